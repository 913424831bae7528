"""What of the tree decoding and the 4-bit weights runs on the host."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def mods():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import best_of_n, qweight, tree_decode
    return best_of_n, qweight, tree_decode


def _refused(gs, f, *args, **kw):
    with pytest.raises(gs.GsError) as e:
        f(*args, **kw)
    assert e.value.code == gs.GS_ERR_INVALID_ARG


def test_trees(mods):
    bn = mods[0]
    nodes, masks, depths = bn.check_trees([(0, 5, [1, 2, 3, 4], [-1, 0, 0, 2]), (3, 0, [9], [7])], 8, 4)
    assert nodes == 4 and masks == [[1, 3, 5, 13], [1, 0, 0, 0]] and depths == [[0, 1, 1, 2], [0, 0, 0, 0]]
    chain = list(range(-1, 63))
    nodes, masks, _ = bn.check_trees([(0, 0, [0] * 64, chain)], 64, 1)
    assert masks[0][63] == 2 ** 64 - 1
    for bad in ([], [(0, 0, [], [])], [(0, 0, [1], [-1]), (1, 0, [], [])], [(0, 0, [0] * 65, [0] * 65)],
                [(0, 0, [1, 2], [-1])], [(0, 0, [1, 2], [-1, 1])], [(0, 0, [1, 2], [-1, -1])],
                [(0, 0, [1, 2], [-1, 2])], [(0, 0, [1], [-1]), (0, 0, [1], [-1])],
                [(0, 0, [1] * 5, [0] * 5), (1, 0, [1], [0])], [(i, 0, [1], [0]) for i in range(5)]):
        _refused(bn.gs, bn.check_trees, bad, 8 if len(bad) != 1 else 70, 4)


@pytest.mark.parametrize("max_nodes,depth,ngram", [(1, 4, 3), (5, 2, 1), (16, 8, 3), (64, 10, 2), (9, 0, 3)])
def test_lookup_tree(mods, max_nodes, depth, ngram):
    """Every path from the root stands in the history, behind a copy of its last token."""
    rng = np.random.default_rng(max_nodes)
    for _ in range(30):
        history = rng.integers(0, 4, rng.integers(1, 60)).tolist()
        tokens, parents = mods[2].lookup_tree(history, max_nodes, depth, ngram)
        assert tokens[0] == history[-1] and parents[0] == -1 and 1 <= len(tokens) <= max_nodes
        runs = {tuple(history[i: i + k]) for i in range(len(history)) for k in range(1, depth + 2)}
        seen = set()
        for i in range(1, len(tokens)):
            assert 0 <= parents[i] < i
            assert (parents[i], tokens[i]) not in seen            # no two alike
            seen.add((parents[i], tokens[i]))
            path, at = [], i
            while at >= 0:
                path.append(tokens[at])
                at = parents[at]
            assert len(path) <= depth + 1 and tuple(path[::-1]) in runs


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize(mods, dtype, group, zeros):
    """Each weight comes back within half a step and what the scale's rounding
    (eps / 2 of up to 15 steps) and the zero's (half a step) add; zero weights exactly."""
    g = torch.Generator().manual_seed(group)
    w = (0.05 * torch.randn(40, 256, generator=g)).to(dtype)
    w[3] = 0
    w[4] = w[4].abs()
    w[5, ::2] = 0
    q, scale, zero = mods[1].quantize(w, group, zeros)
    assert q.dtype == torch.uint8 and q.shape == (40, 128) and scale.shape == (40, 256 // group)
    whole = torch.stack([q & 15, q >> 4], -1).flatten(1).float()
    z = 8.0 if zero is None else zero.float().repeat_interleave(group, 1)
    s = scale.float().repeat_interleave(group, 1)
    back = (whole - z) * s
    steps = (0.5 + 0.5 if zeros else 0.5) + 15 * torch.finfo(dtype).eps / 2
    assert ((back - w.float()).abs() <= steps * s + 1e-12).all()
    assert (back[w == 0] == 0).all()


def test_quantize_refuses(mods):
    _, qw, _ = mods
    w = torch.zeros(4, 128, dtype=torch.float16)
    for bad in ((w.float(), 64), (w[0], 64), (w, 16), (w, 0), (w[:, :96], 64), (w[None], 64)):
        _refused(qw.gs, qw.quantize, *bad)
    for bad in (float("nan"), float("inf"), float("-inf")):
        broken = w.clone()
        broken[2, 100] = bad
        _refused(qw.gs, qw.quantize, broken, 64)
    q, s, _ = qw.quantize(w)
    _refused(qw.gs, qw.QWeight, q, s, group=64)                  # not on a device
    _refused(qw.gs, qw.QWeight, q[0], s, group=64)
    _refused(qw.gs, qw.QWeight, q[0, 0], s, group=64)


def test_tree_decode_refuses(mods):
    bn, _, td = mods

    class Dec:
        max_rows = 32

        class pool:
            class table:
                max_ctx = 50
    for bad in (dict(prompts=[]), dict(prompts=[[1], []]), dict(new=0), dict(max_nodes=0),
                dict(max_nodes=65), dict(prompts=[[1]] * 3), dict(prompts=[[1] * 45]), dict(new=50)):
        a = {**dict(prompts=[[1, 2], [3]], new=10, max_nodes=16), **bad}
        _refused(bn.gs, td.tree_decode, Dec, a.pop("prompts"), a.pop("new"), **a)
