"""gs_tree_accept and gs_tree_commit: whole numbers and moves, so everything is exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.int32).to(DEV)


def _walk(parent, token, choice, count, most, eos):
    path, at = [], 0
    while count > 0 and len(path) < most:
        path.append(at)
        want = choice[at]
        if want < 0 or want == eos:
            break
        kids = [i for i in range(1, count) if parent[i] == at and token[i] == want]
        if not kids:
            break
        at = kids[0]
    return path


def _trees(rng, trees, nodes, vocab, hit):
    """Random trees; with a vocabulary of few tokens siblings often carry the same one."""
    parent = np.array([[-1] + [rng.integers(0, i) for i in range(1, nodes)] for _ in range(trees)])
    token = rng.integers(0, vocab, (trees, nodes))
    choice = rng.integers(-1, vocab, (trees, nodes))
    for b in range(trees):
        for i in rng.permutation(np.arange(1, nodes)):
            if rng.random() < hit:
                choice[b, parent[b, i]] = token[b, i]
    return parent, token, choice


def _accept(gs, parent, token, choice, count=None, most=None, eos=-1, stream=None):
    trees, nodes = parent.shape
    t = [_dev(x) for x in (parent, token, choice)]
    opt = [None if x is None else _dev(x) for x in (count, most)]
    path = torch.full((trees, nodes), 99, dtype=torch.int32, device=DEV)
    new, length = torch.full_like(path, 99), torch.full((trees,), 99, dtype=torch.int32, device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    gs.gs_tree_accept(*[x.data_ptr() for x in t], *[0 if x is None else x.data_ptr() for x in opt], eos,
                      trees, nodes, path.data_ptr(), new.data_ptr(), length.data_ptr(), err.data_ptr(),
                      (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return path.cpu().numpy(), new.cpu().numpy(), length.cpu().numpy(), int(err.item())


def _check(got, parent, token, choice, count=None, most=None, eos=-1):
    trees, nodes = parent.shape
    path, new, length, _ = got
    for b in range(trees):
        c = nodes if count is None else min(max(int(count[b]), 0), nodes)
        m = nodes if most is None else int(most[b])
        want = _walk(parent[b].tolist(), token[b].tolist(), choice[b].tolist(), c, m, eos)
        rest = [-1] * (nodes - len(want))
        assert length[b] == len(want)
        assert path[b].tolist() == want + rest
        assert new[b].tolist() == [choice[b, i] for i in want] + rest


@pytest.mark.parametrize("nodes", [1, 2, 3, 17, 31, 32, 33, 47, 63, 64])
@pytest.mark.parametrize("trees", [1, 5, 130])
def test_paths(gs, nodes, trees):
    rng = np.random.default_rng(nodes * 1000 + trees)
    for vocab, hit in ((2, 0.9), (4, 0.7), (1000, 0.95), (1000, 0.0)):
        t = _trees(rng, trees, nodes, vocab, hit)
        got = _accept(gs, *t, stream=torch.cuda.Stream())
        assert got[3] == 0
        _check(got, *t)
        count, most = rng.integers(0, nodes + 1, trees), rng.integers(-1, nodes + 2, trees)
        got = _accept(gs, *t, count=count, most=most, eos=1)
        assert got[3] == 0
        _check(got, *t, count=count, most=most, eos=1)


def test_chains_of_every_length(gs):
    """A chain of 64 nodes that agrees up to node b."""
    nodes = 64
    parent = np.tile(np.arange(nodes) - 1, (nodes, 1))
    token = np.tile(np.arange(nodes) + 100, (nodes, 1))
    choice = token + 1
    choice[np.arange(nodes), np.arange(nodes)] = 7
    got = _accept(gs, parent, token, choice)
    assert got[2].tolist() == list(range(1, nodes + 1))
    _check(got, parent, token, choice)


def test_of_equal_siblings_the_first(gs):
    """Children of one node with the same token, on both sides of node 32."""
    nodes = 64
    parent, token, choice = np.zeros((3, 1, nodes), np.int64)
    token[0], choice[0] = 5, 5
    for first in (1, 2, 31, 32, 33, 40, 63):
        token[0, 1:first] = 6
        token[0, first:] = 5
        parent[0, first + 1:] = 0
        choice[0, first] = 8
        got = _accept(gs, parent, token, choice)
        _check(got, parent, token, choice)
        assert got[0][0, :3].tolist() == ([0, first, -1])
        choice[0, first] = 5


def test_accept_error_word(gs):
    """A parent that is not a lower number, or a bad count: the node is on no path."""
    rng = np.random.default_rng(3)
    parent, token, choice = _trees(rng, 3, 40, 3, 0.9)
    for bad in (-1, 20, 21, 63, 2 ** 31 - 1, -2 ** 31):
        p, c = parent.copy(), choice.copy()
        p[1, 20] = bad
        got = _accept(gs, p, token, c)
        assert got[3] == 1
        q, t = p.copy(), token.copy()
        q[1, 20], t[1, 20] = 0, -5                       # never chosen
        _check(got, q, t, c)
    for bad in (-1, 41):
        count = np.array([40, bad, 40])
        got = _accept(gs, parent, token, choice, count=count)
        assert got[3] == 1
        _check(got, parent, token, choice, count=count)


# -------------------------------------------------------------------- commit
def _pool(rng, layers, ns, nodes, Hkv, D, spare=3):
    per = -(-(max(ns) + nodes) // 64)
    pages = len(ns) * per + spare
    pool = torch.from_numpy(rng.integers(-30000, 30000, (layers, pages, 2, Hkv, 64 * D), dtype=np.int16)).to(DEV)
    table = rng.permutation(pages)[: len(ns) * per].reshape(len(ns), per)
    return pool, table


def _moved(pool, table, ns, path, length, Hkv, D):
    want = pool.clone()
    k, v = ([p.view(*pool.shape[:3], Hkv, *s) for p in (pool, want)] for s in ((64, D), (D, 64)))
    for b, n in enumerate(ns):
        for i in range(int(length[b])):
            src, dst = n + int(path[b, i]), n + i
            ps, pd = int(table[b, src // 64]), int(table[b, dst // 64])
            k[1][:, pd, 0, :, dst % 64] = k[0][:, ps, 0, :, src % 64]
            v[1][:, pd, 1, :, :, dst % 64] = v[0][:, ps, 1, :, :, src % 64]
    return want


def _commit(gs, pool, table, ns, path, length, Hkv, D, seq=None, bf16=False, stream=None):
    t = [_dev(x) for x in (np.array(ns), path, length, table)]
    s = None if seq is None else _dev(seq)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = gs.gs_cache(pool.data_ptr(), pool.shape[1], Hkv, D, gs.GS_BF16 if bf16 else gs.GS_F16,
                        t[3].data_ptr(), table.shape[0], table.shape[1])
    torch.cuda.synchronize()
    gs.gs_tree_commit(cache, pool.shape[0], 0 if s is None else s.data_ptr(), t[0].data_ptr(),
                      t[1].data_ptr(), t[2].data_ptr(), path.shape[0], path.shape[1], err.data_ptr(),
                      (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return int(err.item())


def _paths(rng, trees, nodes):
    length = rng.integers(0, nodes + 1, trees)
    length[0] = nodes
    path = np.full((trees, nodes), -1)
    for b, m in enumerate(length):
        path[b, :m] = np.sort(rng.permutation(nodes)[:m])
    return path, length


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes", [1, 2, 5, 17, 33, 48, 64])
@pytest.mark.parametrize("Hkv,layers", [(1, 1), (3, 4)])
def test_moves(gs, D, nodes, Hkv, layers):
    """Rising paths of every kind, over page borders, in every layer; nothing else moves."""
    rng = np.random.default_rng(nodes + D)
    ns = [0, 1, 30, 63, 64, 65, 100, 127, 128, 700]
    for _ in range(3):
        pool, table = _pool(rng, layers, ns, nodes, Hkv, D)
        path, length = _paths(rng, len(ns), nodes)
        want = _moved(pool, table, ns, path, length, Hkv, D)
        assert _commit(gs, pool, table, ns, path, length, Hkv, D, bf16=D == 128,
                       stream=torch.cuda.Stream()) == 0
        assert torch.equal(pool, want)


def test_every_number_of_moved_tokens(gs):
    """One to 63 tokens move, from next door or from the tree's end."""
    rng = np.random.default_rng(1)
    ns = [40] * 63
    for far in (False, True):
        path = np.full((63, 64), -1)
        length = np.arange(1, 64)
        for m in length:
            path[m - 1, :m] = np.arange(m) + (64 - m if far else 1)
        pool, table = _pool(rng, 2, ns, 64, 2, 64)
        want = _moved(pool, table, ns, path, length, 2, 64)
        assert _commit(gs, pool, table, ns, path, length, 2, 64) == 0
        assert torch.equal(pool, want)


def test_other_sequences_and_offsets_past_32_bits(gs):
    """Trees of sequences in another order; layers and pages far into the pool."""
    rng = np.random.default_rng(2)
    Hkv, D = 8, 128
    page = 2 * Hkv * 64 * D
    pages = 2 ** 31 // page + 20
    pool = torch.zeros(2, pages, 2, Hkv, 64 * D, dtype=torch.int16, device=DEV)
    table = np.array([[pages - 1, pages - 3], [pages - 2, 5], [7, pages - 4]])
    for p in np.unique(table):
        pool[:, p] = torch.from_numpy(rng.integers(-30000, 30000, (2, 2, Hkv, 64 * D), dtype=np.int16)).to(DEV)
    ns, seq = [50, 20], np.array([2, 0])
    path, length = _paths(rng, 2, 40)
    small = np.unique(table)
    want = _moved(pool[:, small], np.searchsorted(small, table[seq]), ns, path, length, Hkv, D)
    assert _commit(gs, pool, table, ns, path, length, Hkv, D, seq=seq) == 0
    assert torch.equal(pool[:, small], want)


@pytest.mark.parametrize("room", [1, 5, 16])
def test_paths_that_end_with_the_table(gs, room):
    """A tree of few nodes at the end of its table, beside a wider one."""
    rng = np.random.default_rng(room)
    pool, table = _pool(rng, 2, [100, 100], 20, 2, 64)
    ns = [64 * table.shape[1] - room, 30]
    path, length = _paths(rng, 2, 20)
    path[0], length[0] = -1, (room + 1) // 2
    path[0, : length[0]] = np.arange(room)[room % 2 == 0:: 2]      # its last node is the table's last
    want = _moved(pool, table, ns, path, length, 2, 64)
    assert _commit(gs, pool, table, ns, path, length, 2, 64) == 0
    assert torch.equal(pool, want)


def test_commit_error_word(gs):
    """What is out of range raises the word; nothing of that tree moves, the others do."""
    rng = np.random.default_rng(4)
    ns, nodes, Hkv, D = [10, 70, 130], 9, 2, 64
    for what in ("length", "long", "falls", "twice", "node", "negative", "seq", "n", "far", "page"):
        pool, table = _pool(rng, 2, ns, nodes, Hkv, D)
        path = np.tile(np.array([0, 2, 3, 5, 8, -1, -1, -1, -1]), (3, 1))
        length, seq, n = np.array([5, 5, 5]), np.arange(3), np.array(ns)
        want = _moved(pool, table, ns, path, np.array([5, 0, 5]), Hkv, D)
        if what == "length":
            length[1] = -1
        elif what == "long":
            length[1] = 10
        elif what == "falls":
            path[1, 3] = 1
        elif what == "twice":
            path[1, 3] = 3
        elif what == "node":
            path[1, 4] = 9
        elif what == "negative":
            path[1, 0] = -1
        elif what == "seq":
            seq[1] = 3
        elif what == "n":
            n[1] = -1
        elif what == "far":
            n[1] = 64 * table.shape[1] - 8
        else:
            table[1, 1] = pool.shape[1]
        assert _commit(gs, pool, table, n, path, length, Hkv, D, seq=seq) == 1, what
        assert torch.equal(pool, want), what
