"""gs_tree_attention with more than eight tiles of 128 query rows to a KV head, whose blocks form
several teams, and trees of fewer tiles than a team has blocks.  Tolerances as in
test_gpu_tree_attention."""
import pytest

from tests.test_gpu_tree_attention import NS, _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("bf16", 64), ("fp16", 128), ("bf16", 128)])
@pytest.mark.parametrize("nodes,Hq,Hkv", [(64, 40, 1), (64, 20, 1), (61, 40, 2), (64, 17, 1), (33, 72, 1)])
def test_many_tiles(gs, dtype, D, nodes, Hq, Hkv):
    c = _case(dtype, NS, nodes, Hq, Hkv, D, seed=nodes + Hq + D)
    for split in (0, 1, 5):
        out, lse, err = _run(gs, c, split=split, all_nodes=True)
        assert err == 0
        _check(c, out, lse)


@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("bf16", 128)])
@pytest.mark.parametrize("nodes,Hq,Hkv", [(64, 40, 1), (64, 40, 2), (64, 6, 1)])
def test_trees_of_fewer_tiles(gs, dtype, D, nodes, Hq, Hkv):
    """Counts that leave some blocks of a team without a tile, with any mask and with windows."""
    counts = [nodes, 0, 1, 3, nodes - 1, 7, nodes, 20, 2, 40, nodes // 3]
    for masks, window in (("any", 0), ("tree", 0), ("tree", 50), ("any", 300)):
        c = _case(dtype, NS, nodes, Hq, Hkv, D, seed=nodes, counts=counts, masks=masks)
        out, lse, err = _run(gs, c, window=window)
        assert err == 0
        _check(c, out, lse, window)


@pytest.mark.parametrize("nodes,Hq,Hkv", [(64, 40, 1), (64, 24, 2)])
def test_one_long_sequence(gs, nodes, Hq, Hkv):
    """Every team's share of one tree, and parts of the tiles that teams divide."""
    c = _case("bf16", [9000], nodes, Hq, Hkv, 128, seed=1)
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)
    again, l2, _ = _run(gs, c)
    assert (again == out).all() and (l2 == lse).all()
