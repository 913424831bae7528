"""gs_tree_attention against masked softmax attention in 64 bits.

Tolerances.  With A = sum_j p_j |v_j| of a row, an output carries the rounding
of the probabilities to the cache's type (u A, u = 2^-11 in fp16 and 2^-8 in
bf16), its own rounding (u |o|, at most u A), and the fp32 arithmetic: scores
of up to 128 products (relative 2^-24 each, scores of size at most about 30)
shift a probability by at most 3e-5: 2.1 u A + 1e-4 A bounds the sum.  The
log-sum-exp carries the scores' error only: 5e-5."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
KEPT = 7.0                   # what rows that are not in use hold


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _cache(gs, pool, table, Hkv, D, dtype):
    return gs.gs_cache(pool.data_ptr(), pool.shape[0], Hkv, D,
                       gs.GS_F16 if dtype == "fp16" else gs.GS_BF16, table.data_ptr(),
                       table.shape[0], table.shape[1])


def _tree_masks(rng, trees, nodes):
    """Ancestors of trees whose nodes hang on any earlier one; and their depths."""
    mask, depth = np.zeros((trees, nodes), np.uint64), np.zeros((trees, nodes), np.int64)
    for b in range(trees):
        for i in range(nodes):
            mask[b, i] = np.uint64(1 << i)
            if i:
                up = rng.integers(0, i)
                mask[b, i] |= mask[b, up]
                depth[b, i] = depth[b, up] + 1
    return mask, depth


def _case(dtype, ns, nodes, Hq, Hkv, D, seed, counts=None, masks="tree", stride=None, spare=2,
          stretch=1.0):
    """Keys and values of each sequence and its tree, in shuffled pages; whatever a
    page holds beyond a tree's keys, and every spare page, is NaN."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, B = TYPES[dtype], len(ns)
    counts = [nodes] * B if counts is None else counts
    per = max(1, -(-max(n + c for n, c in zip(ns, counts)) // 64)) if stride is None else stride
    n_pages = B * per + spare
    table = rng.permutation(n_pages)[: B * per].reshape(B, per)
    pool = torch.full((n_pages, 2, Hkv, 64 * D), float("nan"), dtype=dt, device=DEV)
    ks, vs = [], []
    for b in range(B):
        n = ns[b] + counts[b]
        k = (stretch * torch.randn(n, Hkv, D, device=DEV, generator=g)).to(dt)
        v = torch.randn(n, Hkv, D, device=DEV, generator=g).to(dt)
        t = torch.arange(n, device=DEV)
        pg = torch.from_numpy(table[b]).to(DEV)[t // 64]
        pool.view(-1, 2, Hkv, 64, D)[pg, 0, :, t % 64] = k
        pool.view(-1, 2, Hkv, D, 64)[pg, 1, :, :, t % 64] = v
        ks.append(k)
        vs.append(v)
    mask, depth = _tree_masks(rng, B, nodes)
    if masks == "any":       # any pattern, bits beyond the nodes and empty rows among them
        mask = rng.integers(0, 2 ** 64, (B, nodes), dtype=np.uint64)
        mask[:, ::3] = 0
        mask[:, 1::5] = np.uint64(2 ** 64 - 1)
    q = (2 * torch.randn(B, nodes, Hq, D, device=DEV, generator=g)).to(dt)
    return dict(dtype=dtype, ns=list(ns), nodes=nodes, counts=list(counts), Hq=Hq, Hkv=Hkv, D=D, pool=pool,
                k=ks, v=vs, q=q, mask=mask, pos=np.asarray(ns)[:, None] + depth,
                table=torch.from_numpy(table.astype(np.int32)).to(DEV))


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _run(gs, c, window=0, split=0, seq=None, only=None, q=None, ld=None, stream=None, scratch=None,
         lse=True, all_nodes=False, n=None, count=None):
    """Outputs, log-sum-exps and the error word; `only`: these trees, in this order."""
    D, Hq, nodes = c["D"], c["Hq"], c["nodes"]
    pick = list(range(len(c["ns"]))) if only is None else only
    B = len(pick)
    q = c["q"][pick].reshape(B * nodes, -1).contiguous() if q is None else q
    n = _dev(np.array(c["ns"])[pick]) if n is None else n
    count = (None if all_nodes else _dev(np.array(c["counts"])[pick])) if count is None else count
    mask, pos = _dev(c["mask"][pick].view(np.int64), torch.int64), _dev(c["pos"][pick])
    if seq is None and only is not None:
        seq = _dev(np.array(pick))
    out = torch.full((B * nodes, ld or Hq * D), KEPT, dtype=q.dtype, device=DEV)
    ls = torch.full((B * nodes, Hq), KEPT, device=DEV)
    cache = _cache(gs, c["pool"], c["table"], c["Hkv"], D, c["dtype"])
    nb = gs.gs_tree_attention_scratch_bytes(cache, B, nodes, Hq, split)
    assert nb >= 256
    if scratch is None:      # stale bytes everywhere but in the error word
        scratch = torch.full((nb,), 0x7F, dtype=torch.uint8, device=DEV)
        scratch[:4] = 0
    torch.cuda.synchronize()
    gs.gs_tree_attention(cache, q.data_ptr(), q.stride(0), 0 if seq is None else seq.data_ptr(),
                         n.data_ptr(), 0 if count is None else count.data_ptr(), mask.data_ptr(),
                         pos.data_ptr() if window else 0, B, nodes, Hq, D ** -0.5, window,
                         out.data_ptr(), out.stride(0), ls.data_ptr() if lse else 0, split,
                         scratch.data_ptr(), scratch.numel(),
                         (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return out, ls, int(scratch[:4].view(torch.int32).item())


def _seen(c, b, window):
    n, m = c["ns"][b], c["counts"][b]
    see = np.zeros((m, n + m), bool)
    for i in range(m):
        lo = min(n, max(0, max(int(c["pos"][b][i]), n) + 1 - window)) if window else 0
        see[i, lo:n] = True
        see[i, n:] = [(int(c["mask"][b, i]) >> j) & 1 for j in range(m)]
    return torch.from_numpy(see).to(DEV)


def _check(c, out, lse, window=0, trees=None, slack=1e-4, lse_slack=5e-5):
    Hq, Hkv, D, nodes = c["Hq"], c["Hkv"], c["D"], c["nodes"]
    u = UNIT[c["dtype"]]
    for b in range(len(c["ns"])) if trees is None else trees:
        m = c["counts"][b]
        o, l = out.view(-1, nodes, out.shape[1])[b], lse.view(-1, nodes, Hq)[b]
        assert (o[m:] == KEPT).all() and (l[m:] == KEPT).all()
        if m == 0:
            continue
        o, l = o[:m, : Hq * D].double().view(m, Hkv, -1, D), l[:m].double()
        assert torch.isfinite(o).all()
        see = _seen(c, b, window)
        k, v = c["k"][b].double(), c["v"][b].double()
        s = torch.einsum("thgd,nhd->thgn", c["q"][b, :m].double().view(m, Hkv, -1, D), k) * D ** -0.5
        s = s.masked_fill(~see[:, None, None], float("-inf"))
        p = torch.softmax(s, -1).nan_to_num(0.0)           # (a row that sees nothing)
        want = torch.einsum("thgn,nhd->thgd", p, v)
        bound = (2.1 * u + slack) * torch.einsum("thgn,nhd->thgd", p, v.abs()) + 2.0 ** -24
        bound[~see.any(1)] = 0.0
        worst = ((o - want).abs() - bound).max().item()
        assert worst <= 0.0, (b, c["ns"][b], worst)
        ref = torch.logsumexp(s, -1).view(m, -1)
        empty = ~see.any(1)
        assert (l[empty] == float("-inf")).all()
        assert (l[~empty] - ref[~empty]).abs().max().item() <= lse_slack if (~empty).any() else True


NS = [0, 1, 31, 32, 47, 63, 64, 65, 130, 511, 700]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes,Hq,Hkv", [(1, 4, 4), (2, 16, 2), (5, 16, 8), (17, 4, 2), (17, 3, 1),
                                          (33, 8, 1), (63, 5, 1), (64, 4, 4), (64, 16, 2), (9, 40, 1), (64, 12, 1)])
def test_lengths_nodes_and_groups(gs, dtype, D, nodes, Hq, Hkv):
    c = _case(dtype, NS, nodes, Hq, Hkv, D, seed=nodes + Hq + D)
    out, lse, err = _run(gs, c, all_nodes=True)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("bf16", 128)])
@pytest.mark.parametrize("nodes,Hq,Hkv", [(7, 4, 2), (40, 8, 4), (64, 2, 1), (64, 8, 1), (60, 10, 1)])
def test_any_mask_and_counts(gs, dtype, D, nodes, Hq, Hkv):
    """Any pattern of bits, nodes that see nothing, trees of fewer nodes, of none."""
    counts = [nodes, 0, 1, nodes // 2, nodes - 1, nodes, nodes, 3, nodes, 0, nodes // 3]
    c = _case(dtype, NS, nodes, Hq, Hkv, D, seed=nodes, counts=counts, masks="any")
    for split in (0, 1):
        out, lse, err = _run(gs, c, split=split)
        assert err == 0
        _check(c, out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [1, 2, 20, 63, 64, 65, 100, 640, 5000, 2 ** 31 - 1])
def test_window(gs, D, window):
    """Each node's window starts at its own position; keys that no node sees are NaN."""
    ns = [0, 1, 64, 65, 200, 777, 1290]
    c = _case("bf16", ns, 12, 8, 2, D, seed=window % 1000)
    t = c["table"].cpu().numpy()
    for b, n in enumerate(ns):
        for j in range(max(0, min(n, n + 1 - window))):
            page = int(t[b, j // 64])
            c["pool"].view(-1, 2, 2, 64, D)[page, 0, :, j % 64] = float("nan")
            c["pool"].view(-1, 2, 2, D, 64)[page, 1, :, :, j % 64] = float("nan")
    for split in (0, 1, 3):
        out, lse, err = _run(gs, c, window=window, split=split)
        assert err == 0
        _check(c, out, lse, window)


def test_window_positions_below_the_length_count_as_it(gs):
    c = _case("fp16", [300, 500], 6, 4, 2, 64, seed=3)
    c["pos"] = c["pos"] - 1000
    c["pos"][1, 2:] = 2 ** 31 - 1                            # sees no cached key
    out, lse, err = _run(gs, c, window=70)
    assert err == 0
    _check(c, out, lse, 70)


@pytest.mark.parametrize("split", [1, 2, 5, 40, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("nodes", [3, 20, 64])
def test_splits(gs, split, nodes):
    """Any division of the length, the joining kernel's many items included."""
    c = _case("fp16", [4500, 64, 0, 321], nodes, 8, 2, 64, seed=split % 100)
    out, lse, err = _run(gs, c, split=split)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("D,nodes", [(128, 4), (64, 30), (128, 40)])
def test_long_pages_per_warp(gs, D, nodes):
    """More than 32 pages for one warp (its page numbers are read in groups of 32)."""
    c = _case("fp16", [20000], nodes, 2, 1, D, seed=4)
    out, lse, err = _run(gs, c, split=400)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("nodes", [5, 33])
def test_trees_do_not_depend_on_the_batch(gs, nodes):
    """With a given split a tree's bits are its own: alone, in a batch, in another order."""
    ns = [1, 640, 1999, 130]
    c = _case("fp16", ns, nodes, 16, 8, 64, seed=8, stride=40)
    out, lse, _ = _run(gs, c, split=4)
    out, lse = out.view(4, nodes, -1), lse.view(4, nodes, -1)
    order = [2, 0, 3, 1]
    o2, l2, _ = _run(gs, c, split=4, only=order)
    assert torch.equal(o2.view(4, nodes, -1), out[order]) and torch.equal(l2.view(4, nodes, -1), lse[order])
    for b in range(4):
        o1, l1, _ = _run(gs, c, split=4, only=[b])
        assert torch.equal(o1, out[b]) and torch.equal(l1, lse[b])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes", [4, 24])
def test_ways_of_joining_give_the_same_bits(gs, D, nodes):
    """Few trees join their items within a cluster, many through the scratch."""
    ns = [1500, 300, 64, 0, 1, 1950] * 8
    c = _case("bf16", ns, nodes, 8, 8, D, seed=D)
    out, lse, err = _run(gs, c, split=8)
    assert err == 0
    _check(c, out, lse, trees=range(6))
    out, lse = out.view(len(ns), nodes, -1), lse.view(len(ns), nodes, -1)
    for b in range(6):
        o1, l1, _ = _run(gs, c, split=8, only=[b])
        assert torch.equal(o1, out[b]) and torch.equal(l1, lse[b])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nodes,Hq", [(6, 2), (30, 2), (48, 8)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_that_are_not_finite_reach_only_their_own(gs, D, nodes, Hq, bad):
    """A node's key and value that are not finite: nodes that do not see it are as before."""
    c = _case("fp16", [90, 0, 63], nodes, Hq, 2, D, seed=nodes)
    base, base_lse, _ = _run(gs, c)
    t = c["table"].cpu().numpy()
    victim = [2, 4, nodes - 1]
    for b, j in enumerate(victim):
        slot = c["ns"][b] + j
        page = int(t[b, slot // 64])
        c["pool"].view(-1, 2, 2, D, 64)[page, 1, 1, ::7, slot % 64] = bad     # one KV head's
    out, lse, err = _run(gs, c)
    assert err == 0 and torch.equal(lse, base_lse)
    sees = torch.stack([_dev((c["mask"][b] >> np.uint64(j)) & np.uint64(1) > 0, torch.bool)
                        for b, j in enumerate(victim)])
    o, w = (x.view(3, nodes, 2, Hq // 2, D) for x in (out, base))
    assert torch.equal(o[:, :, 0], w[:, :, 0])
    assert torch.equal(o[~sees], w[~sees])
    hit = o[sees][:, 1]
    assert torch.isnan(hit[..., ::7]).all() if bad != bad else (hit[..., ::7] == bad).all()
    rest = [d for d in range(D) if d % 7]
    assert torch.equal(hit[..., rest], w[sees][:, 1][..., rest])
    # keys as well: only the nodes that see it change
    for b, j in enumerate(victim):
        slot = c["ns"][b] + j
        c["pool"].view(-1, 2, 2, 64, D)[int(t[b, slot // 64]), 0, :, slot % 64] = float("nan")
    out, lse, err = _run(gs, c)
    assert err == 0 and torch.equal(out.view(3, nodes, -1)[~sees], base.view(3, nodes, -1)[~sees])
    assert torch.equal(lse.view(3, nodes, -1)[~sees], base_lse.view(3, nodes, -1)[~sees])


@pytest.mark.parametrize("nodes", [3, 20, 64])
def test_windowed_values_that_are_not_finite(gs, nodes):
    """A cached value that only the shallow nodes' windows still reach."""
    window, n = 40, 200
    c = _case("bf16", [n], nodes, 4, 4, 64, seed=5)
    c["pos"] = n + np.arange(nodes)[None] // 2
    base, base_lse, _ = _run(gs, c, window=window)
    at = n + 1 - window + 1                               # seen at positions n and n + 1
    page = int(c["table"][0, at // 64])
    c["pool"].view(-1, 2, 4, 64, 64)[page, 1, :, :, at % 64] = float("inf")
    out, lse, err = _run(gs, c, window=window)
    assert err == 0 and torch.equal(lse, base_lse)
    sees = torch.from_numpy(c["pos"][0] - window < at)
    assert (out[sees] == float("inf")).all() and torch.equal(out[~sees], base[~sees])


def test_one_node_is_one_token(gs):
    """A tree of one node does what gs_decode_attention does for that token."""
    ns = [0, 64, 300, 511, 2000]
    c = _case("fp16", ns, 1, 16, 8, 64, seed=1)
    out, lse, _ = _run(gs, c)
    cache = _cache(gs, c["pool"], c["table"], 8, 64, "fp16")
    o = torch.zeros_like(out)
    l = torch.zeros_like(lse)
    nb = gs.gs_decode_attention_scratch_bytes(cache, 5, 16, 0)
    scratch = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    n = _dev(np.array(ns) + 1)
    gs.gs_decode_attention(cache, c["q"].data_ptr(), 1024, 0, n.data_ptr(), 5, 16, 0.125, 0, o.data_ptr(),
                           1024, l.data_ptr(), 0, scratch.data_ptr(), nb,
                           torch.cuda.current_stream().cuda_stream)
    _check(c, o, l)
    _check(c, out, lse)
    assert (lse - l).abs().max().item() <= 1e-4


def test_shared_pages(gs):
    """Two trees over the same cached pages, each with its own last page."""
    c = _case("bf16", [192, 192], 20, 8, 4, 64, seed=2)
    c["table"][1, :3] = c["table"][0, :3]
    c["k"][1][:192], c["v"][1][:192] = c["k"][0][:192], c["v"][0][:192]
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("nodes", [4, 40])
def test_strides_streams_and_no_lse(gs, nodes):
    c = _case("fp16", [77, 513, 90], nodes, 4, 2, 128, seed=5)
    out, _, _ = _run(gs, c)
    wide = torch.full((3 * nodes, 4 * 128 + 40), float("nan"), dtype=torch.float16, device=DEV)
    wide[:, : 4 * 128] = c["q"].view(3 * nodes, -1)
    o2, l2, _ = _run(gs, c, q=wide, ld=4 * 128 + 8, stream=torch.cuda.Stream(), lse=False)
    assert torch.equal(o2[:, : 4 * 128], out)
    assert (o2[:, 4 * 128:] == KEPT).all() and (l2 == KEPT).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("nodes", [4, 40])
def test_scores_far_apart(gs, dtype, nodes):
    """Scores of several hundred: the running maximum keeps exponentials in range.
    Scores up to 900 in fp32: 900 * 64 * 2^-24 / 8 of error in an exponent at most."""
    c = _case(dtype, [900, 64, 10], nodes, 4, 4, 64, seed=6, stretch=20.0)
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse, slack=2e-3, lse_slack=2e-3)


@pytest.mark.parametrize("nodes", [4, 40])
def test_offsets_past_32_bits(gs, nodes):
    """Pages whose elements lie more than 2^31 elements into the pool."""
    D, Hkv = 128, 8
    c = _case("bf16", [700], nodes, 16, Hkv, D, seed=7, spare=0)
    page = 2 * Hkv * 64 * D
    far = 2 ** 31 // page + 8
    big = torch.empty(far + c["pool"].shape[0], 2, Hkv, 64 * D, dtype=torch.bfloat16, device=DEV)
    big[far:] = c["pool"]
    c["pool"], c["table"] = big, c["table"] + far
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("nodes,trees", [(2, 1500), (20, 1024), (20, 1025), (33, 1300)])
def test_many_trees(gs, nodes, trees):
    """More trees than the wide kernel shares out, and as many; short, of a few sequences."""
    c = _case("bf16", [3, 0, 70, 129, 64, 31, 200], nodes, 4, 2, 64, seed=trees)
    pick = np.random.default_rng(trees).integers(0, 7, trees).tolist()
    out, lse, err = _run(gs, c, only=pick)
    assert err == 0
    first = {}
    for i, b in enumerate(pick):
        first.setdefault(b, i)
    rows = torch.tensor([first[b] for b in range(7)], device=DEV)
    o, l = out.view(trees, nodes, -1), lse.view(trees, nodes, -1)
    _check(c, o[rows].reshape(7 * nodes, -1), l[rows].reshape(7 * nodes, -1))
    # trees of the same sequence are the same tree: other shares of its pages round otherwise,
    # and both are within the bound above of A, at most the largest value
    same = torch.tensor([first[b] for b in pick], device=DEV)
    most = max(v.abs().max().item() for v in c["v"])
    assert ((o.double() - o[same].double()).abs() <= 2 * (2.1 * UNIT["bf16"] + 1e-4) * most).all()
    if trees > 1024 or nodes == 2:
        assert torch.equal(o, o[same]) and torch.equal(l, l[same])


@pytest.mark.parametrize("nodes", [4, 40])
def test_two_calls_at_once(gs, nodes):
    """Calls on two streams, each with scratch of its own, over one cache."""
    c = _case("fp16", [2000, 70, 900, 1500], nodes, 8, 2, 64, seed=3)
    cache = _cache(gs, c["pool"], c["table"], 2, 64, "fp16")
    n, mask = _dev(np.array(c["ns"])), _dev(c["mask"].view(np.int64), torch.int64)
    qs = [c["q"].reshape(4 * nodes, -1).contiguous(), c["q"].flip(1).reshape(4 * nodes, -1).contiguous()]
    want = [_run(gs, c, q=q, all_nodes=True)[0] for q in qs]
    nb = gs.gs_tree_attention_scratch_bytes(cache, 4, nodes, 8, 0)
    scratch = torch.zeros(2, -(-nb // 256) * 256, dtype=torch.uint8, device=DEV)
    outs = torch.zeros(2, 20, 4 * nodes, 512, dtype=torch.float16, device=DEV)
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for i in range(20):
        for j, st in enumerate(streams):
            gs.gs_tree_attention(cache, qs[j].data_ptr(), 512, 0, n.data_ptr(), 0, mask.data_ptr(), 0, 4, nodes,
                                 8, 0.125, 0, outs[j, i].data_ptr(), 512, 0, 0, scratch[j].data_ptr(), nb,
                                 st.cuda_stream)
    torch.cuda.synchronize()
    for j in range(2):
        assert (outs[j] == want[j]).all()
    assert (scratch[:, :4] == 0).all()


@pytest.mark.parametrize("nodes", [4, 40])
def test_error_word(gs, nodes):
    """A bad sequence, length, count or page raises the word; the other trees are right."""
    for what in ("seq", "long", "negative", "count", "page"):
        c = _case("fp16", [100, 200, 300], nodes, 4, 2, 64, seed=1)
        n, count = _dev(np.array(c["ns"])), _dev(np.array(c["counts"]))
        seq = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
        if what == "seq":
            seq[1] = 3
        elif what == "long":
            n[1] = 64 * c["table"].shape[1] - nodes + 1
        elif what == "negative":
            n[1] = -5
        elif what == "count":
            count[1] = nodes + 1
        else:
            c["table"][1, 2] = c["pool"].shape[0]
        out, lse, err = _run(gs, c, seq=seq, n=n, count=count)
        assert err == 1, what
        _check(c, out, lse, trees=[0, 2])
        if what == "seq":
            assert (out.view(3, nodes, -1)[1] == 0).all()


@pytest.mark.parametrize("nodes,ns", [(5, [517]), (17, [300, 2000, 90]), (40, [900])])
def test_captured_and_replayed(gs, nodes, ns):
    """Two captured graphs that share their scratch, replayed on changed inputs."""
    c = _case("fp16", ns, nodes, 8, 4, 64, seed=9, stride=40)
    cache = _cache(gs, c["pool"], c["table"], 4, 64, "fp16")
    B = len(ns)
    nb = gs.gs_tree_attention_scratch_bytes(cache, B, nodes, 8, 0)
    scratch = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    n, mask = _dev(np.array(ns)), _dev(c["mask"].view(np.int64), torch.int64)
    qs = [torch.zeros(B * nodes, 512, dtype=torch.float16, device=DEV) for _ in range(2)]
    outs = [torch.zeros(B * nodes, 512, dtype=torch.float16, device=DEV) for _ in range(2)]
    graphs = []
    side = torch.cuda.Stream()
    for q, o in zip(qs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            gs.gs_tree_attention(cache, q.data_ptr(), 512, 0, n.data_ptr(), 0, mask.data_ptr(), 0, B, nodes,
                                 8, 0.125, 0, o.data_ptr(), 512, 0, 0, scratch.data_ptr(), nb,
                                 torch.cuda.current_stream().cuda_stream)
        graphs.append(graph)
    for seed in range(2):
        for i, q in enumerate(qs):
            q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed * 2 + i)))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for q, o in zip(qs, outs):
            want, _, _ = _run(gs, c, q=q)
            assert torch.equal(o, want)
