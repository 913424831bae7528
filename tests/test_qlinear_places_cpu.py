"""The hand-over of tensor memory between the products and the additions of gs_qlinear's
kernel for many rows: every order in which its warps can run, walked through.

Parties: two warps that issue the products of every other stage, the tensor cores, which
finish each warp's products in order, and (two of the eight) adding warps.  A group's place may be
overwritten once both have added the group before it, which the issuing warp learns from
a barrier, by the parity of its phases.  Which barrier, and which parity, is the kernel's own
header, compiled here."""
import ctypes
import shutil
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_26638_gb300" / "csrc"
PLACES, ADDERS, RING = 4, 2, 2


@pytest.fixture(scope="module")
def header(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("places")
    (at / "p.cc").write_text(
        f'#include "{CSRC / "qlinear_places.h"}"\n'
        'extern "C" int barrier(int q, int p) { return gs::place_barrier(q, p); }\n'
        'extern "C" int phase(int q, int p) { return gs::place_phase(q, p); }\n')
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", str(at / "p.cc"), "-o", str(at / "p.so")], check=True)
    lib = ctypes.CDLL(str(at / "p.so"))
    return lambda q: lib.barrier(q, PLACES), lambda q: lib.phase(q, PLACES)


def _one_barrier():
    """A barrier a place."""
    return lambda q: q % PLACES, lambda q: q // PLACES % 2


def _walk(per_stage, stages, rule):
    """Every reachable state; returns what goes wrong, or None."""
    barrier, phase = rule
    total = per_stage * stages
    owner = [q // per_stage % 2 for q in range(total)]
    lists = [[q for q in range(total) if owner[q] == w] for w in (0, 1)]
    rank = [lists[owner[q]].index(q) for q in range(total)]
    told, parity = [barrier(q) for q in range(total)], [phase(q) for q in range(total)]

    def passes(count, p):                 # a parity wait: that phase, not the one under way, is the last
        return count % 2 != p

    def steps(state):
        issued, done, adders = state[0:2], state[2:4], state[4:]
        arrived = {}
        for a in adders:                  # 2 q: waits for group q; 2 q + 1: has read it, has not told so
            for q in range(a // 2):
                arrived[told[q]] = arrived.get(told[q], 0) + 1
        for w in (0, 1):
            if issued[w] < len(lists[w]):
                q = lists[w][issued[w]]
                before = q // per_stage - RING          # its operands lie where this stage's did
                ready = before < 0 or done[w] > rank[(before + 1) * per_stage - 1]
                if ready and (q < PLACES or passes(arrived.get(told[q - PLACES], 0) // ADDERS, parity[q - PLACES])):
                    if q >= PLACES and any(a <= 2 * (q - PLACES) for a in adders):
                        yield f"group {q} overwrites group {q - PLACES} before it is added"
                        return
                    yield state[:w] + (issued[w] + 1,) + state[w + 1:]
            if done[w] < issued[w]:
                yield state[:2 + w] + (done[w] + 1,) + state[3 + w:]
        for i, a in enumerate(adders):
            q = a // 2
            if q == total:
                continue
            if a % 2 == 0:
                full = sum(done[owner[r]] > rank[r] for r in range(q % PLACES, total, PLACES))
                if not passes(full, q // PLACES % 2):
                    continue
                if not done[owner[q]] > rank[q]:
                    yield f"group {q} is added before it is there"
                    return
            yield state[:4 + i] + (a + 1,) + state[5 + i:]

    start = (0, 0, 0, 0) + (0,) * ADDERS
    end = (len(lists[0]), len(lists[1])) * 2 + (2 * total,) * ADDERS
    seen, todo = {start}, [start]
    while todo:
        state, found = todo.pop(), False
        for nxt in steps(state):
            found = True
            if isinstance(nxt, str):
                return nxt
            if nxt not in seen:
                seen.add(nxt)
                todo.append(nxt)
        if not found and state != end:
            return "nothing can go on"
    return None if end in seen else "no end"


@pytest.mark.parametrize("group,stages", [(32, 1), (32, 2), (32, 3), (32, 7), (64, 10), (128, 18)])
def test_no_order_loses_a_sum(header, group, stages):
    assert _walk(128 // group, stages, header) is None


def test_the_walk_finds_what_one_barrier_loses():
    """Four groups a stage, one barrier a place: the third stage overwrites the first."""
    assert "overwrites" in _walk(4, 3, _one_barrier())
    assert _walk(4, 2, _one_barrier()) is None
    assert _walk(2, 10, _one_barrier()) is None and _walk(1, 18, _one_barrier()) is None


def test_barriers_are_apart(header):
    """Uses of a place in turn are told on different barriers, all within two a place."""
    barrier, phase = header
    for q in range(200):
        assert 0 <= barrier(q) < 2 * PLACES and barrier(q) != barrier(q + PLACES)
        assert barrier(q) == barrier(q + 2 * PLACES) and phase(q) != phase(q + 2 * PLACES)
    assert len({barrier(q) for q in range(2 * PLACES)}) == 2 * PLACES
