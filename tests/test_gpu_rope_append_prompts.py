"""gs_rope_append on prompts: the sizes at which the host takes other tiles.

On each side of a threshold, with odd remainders:
  values in tiles of 32 tokens instead of 8   from T * Hkv = 4864
  four KV heads to a block of values          from ceil(T / 32) * Hkv = 1216
  eight instead of four heads a lane group    from T * chunks = 9728, with
      chunks = ceil(Hq / (8 hpw)) + ceil(Hkv / (8 hpw)), hpw = 256 / D heads a
      warp; more than 4 hpw query heads then take a second trip of four
Tokens that are not written (slot < 0) lie within runs that would be full.
Tolerances as in test_gpu_rope_append.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_rope_append import DEV, _case, _close, _run, _table, _want

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


CASES = [
    # T, sequences, first slot, Hq, Hkv, D, rot, half, norm
    (4863, 3, 61, 2, 1, 64, 64, True, True),         # tiles of 8
    (4871, 3, 61, 2, 1, 64, 64, True, True),         # tiles of 32
    (1215, 1, 5, 8, 4, 64, 32, False, True),
    (1217, 1, 5, 8, 4, 64, 32, False, True),
    (4832, 4, 1, 8, 8, 64, 64, False, False),        # one KV head to a block of values
    (4833, 4, 1, 8, 8, 64, 64, False, False),        # four
    (4871, 6, 63, 8, 8, 128, 128, True, True),
    (7793, 5, 2, 5, 5, 128, 48, True, True),         # four and one
    (6507, 2, 33, 12, 6, 128, 64, False, True),      # four and two
    (4863, 2, 7, 12, 4, 128, 128, True, True),       # four heads a lane group
    (4871, 2, 7, 12, 4, 128, 128, True, True),       # eight: a second trip, ragged
    (3251, 3, 0, 32, 8, 128, 96, False, True),       # eight, two chunks of query heads
    (4879, 3, 19, 24, 8, 64, 64, True, True),
    (4877, 7, 30, 21, 7, 64, 16, False, False),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("shape", CASES)
def test_prompt(gs, dtype, shape):
    T, seqs, first, Hq, Hkv, D, rot, half, norm = shape
    c = _case(dtype, T, seqs, first, Hq, Hkv, D, seed=T + rot)
    rng = np.random.default_rng(T)
    # not written: single tokens, and one stretch longer than a tile
    gone = np.unique(np.concatenate([rng.integers(0, T, 25), T // 2 + np.arange(45), [0, T - 1]]))
    c["slot"], place = c["slot"].copy(), c["slot"]
    c["slot"][gone] = -1
    rows = int(c["pos"].max()) + 1
    table = _table(gs, rot, rows)
    before = c["pool"].clone()
    rope = gs.gs_rope(table.data_ptr(), rows, rot, gs.ROPE_HALF if half else gs.ROPE_INTERLEAVED)
    q, err = _run(gs, c, rope, norm)
    assert err == 0
    angles = np.arange(rows)[:, None] * (10000.0 ** (-2.0 * np.arange(rot // 2) / rot))[None]
    wq, wk, wv = _want(c, angles, half, norm, rot)
    _close(q.cpu().double().numpy().reshape(T, Hq, D), wq, dtype)
    kept = np.setdiff1d(np.arange(T), gone)
    page, at = c["table"][c["seq"], place // 64][kept], place[kept] % 64
    K = c["pool"].view(-1, 2, Hkv, 64, D)
    V = c["pool"].view(-1, 2, Hkv, D, 64)
    pg, tk = torch.from_numpy(page).to(DEV), torch.from_numpy(at).to(DEV)
    _close(K[pg, 0, :, tk].cpu().double().numpy(), wk[kept], dtype)
    assert np.array_equal(V[pg, 1, :, :, tk].cpu().double().numpy(), wv[kept])
    # nothing else changed
    K[pg, 0, :, tk] = before.view(-1, 2, Hkv, 64, D)[pg, 0, :, tk]
    V[pg, 1, :, :, tk] = before.view(-1, 2, Hkv, D, 64)[pg, 1, :, :, tk]
    assert torch.equal(c["pool"].view(torch.int16), before.view(torch.int16))


def test_thresholds():
    """The cases lie where their comments say."""
    def tiles(T, Hq, Hkv, D):
        hpw = 256 // D
        chunks = -(-Hq // (8 * hpw)) + -(-Hkv // (8 * hpw))
        return (T * Hkv >= 4864, -(-T // 32) * Hkv >= 1216, T * chunks >= 9728)

    got = [tiles(s[0], s[3], s[4], s[5]) for s in CASES]
    assert got[0:2] == [(False, False, False), (True, False, True)]
    assert got[2:4] == [(False, False, False), (True, False, False)]
    assert [g[1] for g in got[4:9]] == [False, True, True, True, True]
    assert [g[2] for g in got[9:]] == [False, True, True, True, True]
    assert len(set(got)) >= 5
