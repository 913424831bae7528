"""gs_decode_attention against softmax attention in 64 bits.

Tolerances.  With A = sum_j p_j |v_j| of a head, an output carries the rounding
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


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _cache(gs, pool, table, Hkv, D, dtype):
    return gs.gs_cache(pool.data_ptr(), pool.shape[0], Hkv, D,
                       gs.GS_F16 if dtype == "fp16" else gs.GS_BF16, table.data_ptr(),
                       table.shape[0], table.shape[1])


def _case(dtype, ns, Hq, Hkv, D, seed, stretch=1.0, spare=2, stride=None):
    """Keys and values of each sequence, in shuffled pages; whatever a page
    holds beyond a sequence's keys, and every spare page, is NaN."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt, B = TYPES[dtype], len(ns)
    per = max(1, -(-max(ns) // 64)) if stride is None else stride
    n_pages = B * per + spare
    table = rng.permutation(n_pages)[: B * per].reshape(B, per)
    pool = torch.full((n_pages, 2, Hkv, 64 * D), float("nan"), dtype=dt, device=DEV)
    ks, vs = [], []
    for b, n in enumerate(ns):
        k = (stretch * torch.randn(n, Hkv, D, device=DEV, generator=g)).to(dt)
        v = torch.randn(n, Hkv, D, device=DEV, generator=g).to(dt)
        t = torch.arange(n, device=DEV)
        pg = torch.from_numpy(table[b]).to(DEV)[t // 64]
        pool.view(-1, 2, Hkv, 64, D)[pg, 0, :, t % 64] = k
        pool.view(-1, 2, Hkv, D, 64)[pg, 1, :, :, t % 64] = v
        ks.append(k)
        vs.append(v)
    q = (2 * torch.randn(B, Hq, D, device=DEV, generator=g)).to(dt)
    return dict(dtype=dtype, ns=ns, Hq=Hq, Hkv=Hkv, D=D, pool=pool, k=ks, v=vs, q=q,
                table=torch.from_numpy(table.astype(np.int32)).to(DEV))


def _run(gs, c, window=0, split=0, seq=None, n=None, q=None, ld=None, scale=None, stream=None,
         scratch=None, lse=True):
    D, Hq = c["D"], c["Hq"]
    q = c["q"].view(len(c["ns"]), -1) if q is None else q
    rows = q.shape[0]
    n = torch.tensor(c["ns"], dtype=torch.int32, device=DEV) if n is None else n
    out = torch.full((rows, ld or Hq * D), float("nan"), dtype=q.dtype, device=DEV)
    ls = torch.full((rows, Hq), float("nan"), device=DEV)
    cache = _cache(gs, c["pool"], c["table"], c["Hkv"], D, c["dtype"])
    nb = gs.gs_decode_attention_scratch_bytes(cache, rows, Hq, split)
    assert nb >= 256
    if scratch is None:      # stale bytes everywhere but in the error word
        scratch = torch.full((nb,), 0x7F, dtype=torch.uint8, device=DEV)
        scratch[:4] = 0
    torch.cuda.synchronize()
    gs.gs_decode_attention(cache, q.data_ptr(), q.stride(0), 0 if seq is None else seq.data_ptr(),
                           n.data_ptr(), rows, Hq, scale or D ** -0.5, window, out.data_ptr(),
                           out.stride(0), ls.data_ptr() if lse else 0, split, scratch.data_ptr(), nb,
                           (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return out, ls, int(scratch[:4].view(torch.int32).item())


def _check(c, out, lse, window=0, rows=None):
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    u = UNIT[c["dtype"]]
    for b, n in enumerate(c["ns"]) if rows is None else rows:
        o = out[b, : Hq * D].double().view(Hkv, Hq // Hkv, D)
        lo = max(0, n - window) if window else 0
        if n == 0:
            assert (o == 0).all() and (lse[b] == float("-inf")).all()
            continue
        k, v = c["k"][b][lo:n].double(), c["v"][b][lo:n].double()
        s = torch.einsum("hgd,nhd->hgn", c["q"][b].double().view(Hkv, -1, D), k) * D ** -0.5
        p = torch.softmax(s, -1)
        want = torch.einsum("hgn,nhd->hgd", p, v)
        bound = (2.1 * u + 1e-4) * torch.einsum("hgn,nhd->hgd", p, v.abs()) + 2.0 ** -24
        worst = ((o - want).abs() / bound).max().item()
        assert worst <= 1.0, (b, n, worst)
        err = (lse[b].double() - torch.logsumexp(s, -1).view(-1)).abs().max().item()
        assert err <= 5e-5, (b, n, err)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (16, 8), (7, 1), (24, 2), (40, 1), (16, 1)])
def test_lengths_and_groups(gs, dtype, D, Hq, Hkv):
    c = _case(dtype, [0, 1, 2, 63, 64, 65, 128, 511, 700, 1025], Hq, Hkv, D, seed=Hq + D)
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 640, 5000, 2 ** 31 - 1])
def test_window(gs, D, window):
    """Keys before the window have no influence: they are NaN."""
    ns = [0, 1, 64, 65, 200, 777, 1290]
    c = _case("bf16", ns, 8, 2, D, seed=window)
    t = c["table"].cpu().numpy()
    for b, n in enumerate(ns):
        for j in range(max(0, n - window)):
            page = int(t[b, j // 64])
            c["pool"].view(-1, 2, 2, 64, D)[page, 0, :, j % 64] = float("nan")
            c["pool"].view(-1, 2, 2, D, 64)[page, 1, :, :, j % 64] = float("nan")
    for split in (0, 1, 3):
        out, lse, err = _run(gs, c, window=window, split=split)
        assert err == 0
        _check(c, out, lse, window)


@pytest.mark.parametrize("split", [1, 2, 5, 40, 1000, 2 ** 31 - 1])
def test_splits(gs, split):
    """Any division of the length, the joining kernel's many items included."""
    c = _case("fp16", [4500, 64, 0, 321], 16, 2, 64, seed=split)
    out, lse, err = _run(gs, c, split=split)
    assert err == 0
    _check(c, out, lse)


def test_long_pages_per_warp(gs):
    """More than 32 pages for one warp (its page numbers are read in groups of 32)."""
    c = _case("fp16", [20000], 2, 1, 128, seed=4)
    out, lse, err = _run(gs, c, split=400)
    assert err == 0
    _check(c, out, lse)


def test_rows_do_not_depend_on_the_batch(gs):
    """With a given split a row's bits are its own: alone, in a batch, in
    another order, with a wider page table."""
    ns = [1, 640, 1999, 130]
    c = _case("fp16", ns, 16, 8, 64, seed=8, stride=40)
    out, lse, _ = _run(gs, c, split=4)
    order = [2, 0, 3, 1]
    seq = torch.tensor(order, dtype=torch.int32, device=DEV)
    q = c["q"].view(4, -1)[order].contiguous()
    n = torch.tensor([ns[i] for i in order], dtype=torch.int32, device=DEV)
    o2, l2, _ = _run(gs, c, split=4, seq=seq, n=n, q=q)
    assert torch.equal(o2, out[order]) and torch.equal(l2, lse[order])
    for b in range(4):
        o1, l1, _ = _run(gs, c, split=4, seq=torch.tensor([b], dtype=torch.int32, device=DEV),
                         n=n.new_tensor([ns[b]]), q=c["q"].view(4, -1)[b: b + 1].contiguous())
        assert torch.equal(o1[0], out[b]) and torch.equal(l1[0], lse[b])


@pytest.mark.parametrize("D", [64, 128])
def test_ways_of_joining_give_the_same_bits(gs, D):
    """Few rows join their items within a cluster, many through the scratch."""
    ns = [1500, 300, 64, 0, 1, 1999] * 8
    c = _case("bf16", ns, 16, 8, D, seed=D)
    out, lse, err = _run(gs, c, split=8)              # 4 items x 8 heads x 48 rows
    assert err == 0
    _check(c, out, lse)
    for b in (0, 1, 2, 3, 4, 5):
        o1, l1, _ = _run(gs, c, split=8, seq=torch.tensor([b], dtype=torch.int32, device=DEV),
                         n=torch.tensor([ns[b]], dtype=torch.int32, device=DEV),
                         q=c["q"].view(len(ns), -1)[b: b + 1].contiguous())
        assert torch.equal(o1[0], out[b]) and torch.equal(l1[0], lse[b])


def test_shared_pages(gs):
    """Two sequences over the same pages, cut at different lengths."""
    c = _case("bf16", [300, 300], 8, 4, 64, seed=2)
    c["table"][1] = c["table"][0]
    c["k"][1], c["v"][1] = c["k"][0], c["v"][0]
    n = torch.tensor([300, 210], dtype=torch.int32, device=DEV)
    out, lse, err = _run(gs, c, n=n)
    assert err == 0
    _check(c, out, lse, rows=[(0, 300), (1, 210)])


def test_strides_streams_and_no_lse(gs):
    c = _case("fp16", [77, 513, 90], 4, 2, 128, seed=5)
    out, _, _ = _run(gs, c)
    wide = torch.full((3, 4 * 128 + 40), float("nan"), dtype=torch.float16, device=DEV)
    wide[:, : 4 * 128] = c["q"].view(3, -1)
    o2, l2, _ = _run(gs, c, q=wide, ld=4 * 128 + 8, stream=torch.cuda.Stream(), lse=False)
    assert torch.equal(o2[:, : 4 * 128], out)
    assert torch.isnan(o2[:, 4 * 128:]).all() and torch.isnan(l2).all()


def test_scores_far_apart(gs):
    """Scores of several hundred, a key of minus infinity, rows whose only
    weight is the last key: the running maximum keeps exponentials in range."""
    c = _case("fp16", [900, 64, 10], 4, 4, 64, seed=6, stretch=20.0)
    out, lse, err = _run(gs, c)
    u = UNIT["fp16"]
    for b, n in enumerate(c["ns"]):
        s = torch.einsum("hgd,nhd->hgn", c["q"][b].double().view(4, 1, 64), c["k"][b].double()) / 8
        p = torch.softmax(s, -1)
        want = torch.einsum("hgn,nhd->hgd", p, c["v"][b].double()).reshape(-1)
        # scores up to 900 in fp32: 900 * 64 * 2^-24 / 8 of error in an exponent at most
        bound = (2.1 * u + 2e-3) * torch.einsum("hgn,nhd->hgd", p, c["v"][b].double().abs()).reshape(-1)
        assert ((out[b].double() - want).abs() <= bound + 2.0 ** -24).all()
        assert torch.allclose(lse[b].double(), torch.logsumexp(s, -1).view(-1), atol=2e-3, rtol=0)


def test_offsets_past_32_bits(gs):
    """Pages whose elements lie more than 2^31 elements into the pool."""
    D, Hkv, n = 128, 8, 700
    c = _case("bf16", [n], 16, Hkv, D, seed=7, spare=0)
    page = 2 * Hkv * 64 * D
    far = 2 ** 31 // page + 8
    big = torch.empty(far + c["pool"].shape[0], 2, Hkv, 64 * D, dtype=torch.bfloat16, device=DEV)
    big[far:] = c["pool"]
    c["pool"], c["table"] = big, c["table"] + far
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)


def test_error_word(gs):
    """A bad sequence, length or page raises the word; the other rows are right."""
    for what in ("seq", "long", "negative", "page"):
        c = _case("fp16", [100, 200, 300], 4, 2, 64, seed=1)
        n = torch.tensor(c["ns"], dtype=torch.int32, device=DEV)
        seq = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
        if what == "seq":
            seq[1] = 3
        elif what == "long":
            n[1] = 64 * c["table"].shape[1] + 1
        elif what == "negative":
            n[1] = -5
        else:
            c["table"][1, 2] = c["pool"].shape[0]
        out, lse, err = _run(gs, c, seq=seq, n=n)
        assert err == 1, what
        _check(c, out, lse, rows=[(0, 100), (2, 300)])
        if what in ("seq", "negative"):
            assert (out[1] == 0).all()
