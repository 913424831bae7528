"""gs_sample against the definition in 64 bits.

A weight is an fp32 exponential of an fp32 argument: its relative error is at
most 2^-24 of the argument's two roundings each time the argument's size (up
to 28) and 2 units of the exponential, 4e-6 in all; so a cumulative share of
the row is known to 4e-6 (DELTA).  A drawn token is right if the interval of
shares that it covers, widened by DELTA, holds the uniform number; a kept count
is right if the cumulative share passes top_p there, to the same DELTA; the
rest (order, ties, top-k counts, greedy rows) is exact."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DELTA = 4e-6
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _run(gs, x, u, stream=None, **par):
    """x: device [rows, vocab] (any row stride); settings as lists or None."""
    rows = x.shape[0]
    dt = {torch.float16: gs.GS_F16, torch.bfloat16: gs.GS_BF16, torch.float32: gs.GS_F32}[x.dtype]
    t = {k: None if par.get(k) is None else torch.tensor(
        par[k], dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV)
        for k in ("temperature", "top_p", "min_p", "top_k")}
    p = gs.gs_sample_params(*[0 if t[k] is None else t[k].data_ptr()
                              for k in ("temperature", "top_p", "min_p", "top_k")])
    u = torch.tensor(u, dtype=torch.float32, device=DEV)
    token = torch.full((rows,), -7, dtype=torch.int32, device=DEV)
    logprob = torch.full((rows,), float("nan"), device=DEV)
    kept = torch.full((rows,), -7, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    gs.gs_sample(x.data_ptr(), x.stride(0), rows, x.shape[1], dt, p, u.data_ptr(), token.data_ptr(),
                 logprob.data_ptr(), kept.data_ptr(),
                 (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return token.cpu().numpy(), logprob.cpu().double().numpy(), kept.cpu().numpy(), u.cpu().double().numpy()


def _check(x, got, temperature=None, top_p=None, min_p=None, top_k=None):
    token, logprob, kept, u = got
    x = x.cpu().double().numpy()
    for r in range(len(x)):
        row = np.where(np.isnan(x[r]), -np.inf, x[r])
        order = np.argsort(-row, kind="stable")
        t = 1.0 if temperature is None else temperature[r]
        if row.max() == -np.inf:
            assert token[r] == -1 and kept[r] == 0 and logprob[r] == -np.inf
            continue
        if not t > 0:
            assert token[r] == order[0] and kept[r] == 1 and logprob[r] == 0
            continue
        s = row[order]
        with np.errstate(invalid="ignore"):
            d = np.where(s == s[0], 0.0, (s - s[0]) / t)
        w = np.where(s == -np.inf, 0.0, np.exp(d))
        w = np.where(w < 2.0 ** -40, 0.0, w)
        n = int((w > 0).sum())
        if min_p is not None and min_p[r] > 0:
            # the count is known up to weights at the threshold itself
            n_lo, n_hi = (int((w >= min(1.0, min_p[r]) * (1 + z)).sum()) for z in (DELTA, -DELTA))
            n_lo = max(n_lo, 1)
        else:
            n_lo = n_hi = n
        if top_k is not None and top_k[r] > 0:
            n_lo, n_hi = min(n_lo, top_k[r]), min(n_hi, top_k[r])
        cum = np.cumsum(w)
        if top_p is not None and top_p[r] < 1:
            total = cum[n_hi - 1]
            assert 1 <= kept[r] <= n_hi
            assert cum[kept[r] - 1] / total >= top_p[r] - DELTA, r
            assert kept[r] == 1 or cum[kept[r] - 2] / total < top_p[r] + DELTA, r
        else:
            # weights within 2^-40 of nothing may or may not count
            slack = int((w[: n_hi + 1] < 2.0 ** -39).sum()) if n_hi == n else 0
            assert n_lo - slack <= kept[r] <= n_hi + slack, (r, kept[r], n_lo, n_hi)
        z = cum[kept[r] - 1]
        at = int(np.flatnonzero(order == token[r])[0])
        assert at < kept[r], (r, at, kept[r])
        uu = min(max(0.0 if np.isnan(u[r]) else u[r], 0.0), 1.0)
        lo, hi = (cum[at] - w[at]) / z, cum[at] / z
        assert lo - DELTA <= uu <= hi + DELTA, (r, lo, uu, hi)
        assert abs(logprob[r] - np.log(w[at] / z)) <= 2 * DELTA, r


def _logits(rows, vocab, seed, dtype, scale=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = scale * torch.randn(rows, vocab, device=DEV, generator=g)
    at = torch.randint(0, vocab, (rows, 4), device=DEV, generator=g)
    x.scatter_add_(1, at, 3 + 6 * torch.rand(rows, 4, device=DEV, generator=g))
    return x.to(TYPES[dtype])


SETTINGS = [
    dict(),
    dict(temperature=0.8),
    dict(top_k=1), dict(top_k=40), dict(top_k=3000),
    dict(top_p=0.9), dict(top_p=0.999), dict(top_p=1e-6), dict(top_p=0.0),
    dict(min_p=0.1), dict(min_p=1.0),
    dict(temperature=1.5, top_k=700, top_p=0.8, min_p=0.001),
    dict(temperature=0.05, top_p=0.95),
    dict(temperature=50.0, top_k=2000, top_p=0.5),      # a nearly flat row
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(5, 59392), (3, 151), (9, 4096), (2, 131071)])
def test_settings(gs, dtype, rows, vocab):
    x = _logits(rows, vocab, vocab + rows, dtype)
    rng = np.random.default_rng(rows)
    for s in SETTINGS:
        par = {k: [v] * rows for k, v in s.items()}
        got = _run(gs, x, rng.random(rows).astype(np.float32), **par)
        _check(x, got, **par)


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 4095, 4097, 32769])
def test_odd_sizes_and_strides(gs, vocab):
    """Rows that start anywhere within a 16-byte vector."""
    for dtype in ("bf16", "fp32"):
        wide = torch.full((6, vocab + 3), 1000.0, dtype=TYPES[dtype], device=DEV)
        wide[:, 1: vocab + 1] = _logits(6, vocab, vocab, dtype) if vocab > 4 else \
            torch.randn(6, vocab, device=DEV).to(TYPES[dtype])
        x = wide[:, 1: vocab + 1]
        par = dict(temperature=[1.0] * 6, top_k=[0, 1, 2, 3, 50, 0], top_p=[0.9, 1.0, 0.5, 1.0, 0.7, 1.0])
        _check(x, _run(gs, x, [0.0, 0.1, 0.5, 0.77, 0.9, 0.9999999], **par), **par)


def test_many_rows(gs):
    """One block, or few, for each row; every row has settings of its own."""
    rows, vocab = 700, 20011
    x = _logits(rows, vocab, 1, "bf16")
    rng = np.random.default_rng(5)
    par = dict(temperature=rng.choice([0.0, 0.3, 1.0, 2.0], rows).tolist(),
               top_k=rng.choice([0, 1, 50, 600], rows).tolist(),
               top_p=rng.choice([1.0, 0.95, 0.4], rows).tolist(),
               min_p=rng.choice([0.0, 0.02], rows).tolist())
    _check(x, _run(gs, x, rng.random(rows).astype(np.float32), **par), **par)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_ties(gs, dtype):
    """Equal logits are ordered by index: a flat row, rows of few distinct
    values (more equal ones than the search gathers), a hot nearly flat row."""
    vocab = 50001
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.zeros(5, vocab, device=DEV)
    x[1] = torch.randint(0, 3, (vocab,), device=DEV, generator=g).float()
    x[2] = torch.randint(-4, 2, (vocab,), device=DEV, generator=g) * 1e-3
    x[3] = 1e-4 * torch.randn(vocab, device=DEV, generator=g)
    x[4, 100] = 0.25
    x = x.to(TYPES[dtype])
    for s in (dict(), dict(top_k=777), dict(top_k=40000), dict(top_p=0.3), dict(min_p=0.5),
              dict(top_k=1000, top_p=0.63)):
        par = {k: [v] * 5 for k, v in s.items()}
        for u in (0.0, 0.123456, 0.5, 0.87654, 0.99999994):
            _check(x, _run(gs, x, [u] * 5, **par), **par)
    # a flat row: the token is floor(u * vocab), exactly
    u = np.float32(0.123456)
    token, _, kept, _ = _run(gs, x[:1], [float(u)])
    assert token[0] == int(float(u) * vocab) and kept[0] == vocab
    token, _, kept, _ = _run(gs, x[:1], [0.99], top_k=[5000])
    assert kept[0] == 5000 and token[0] == int(float(np.float32(0.99)) * 5000)


@pytest.mark.parametrize("rows", [1, 5, 200])
def test_top_p_between_close_totals(gs, rows):
    """Nearly flat rows, where a token weighs less than an estimate of the row's
    mass may be off: top-p ends within and behind the tokens that are noted."""
    vocab = 59392
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = (0.02 * torch.randn(rows, vocab, device=DEV, generator=g)).to(torch.float32)
    rng = np.random.default_rng(rows)
    for p in (0.001, 0.01, 0.03, 0.055, 0.06, 0.3, 0.999):
        par = dict(top_p=[p] * rows)
        _check(x, _run(gs, x, rng.random(rows).astype(np.float32), **par), **par)


def test_masked_and_infinite_logits(gs):
    """-inf and the type's lowest value are never drawn next to ordinary
    logits; NaN counts as -inf; +inf takes the row; a row of -inf gives -1."""
    x = _logits(7, 1000, 4, "fp32")
    x[0, ::2] = float("-inf")
    x[1, :] = float("-inf")
    x[1, 617] = -50.0
    x[2, :] = float("-inf")
    x[3, 5::7] = float("nan")
    x[4, 11] = float("inf")
    x[5, :] = float("nan")
    x[6, 1:] = torch.finfo(torch.float32).min
    rng = np.random.default_rng(0)
    for s in (dict(), dict(top_p=0.9), dict(top_k=600), dict(temperature=0.0), dict(min_p=0.01)):
        par = {k: [v] * 7 for k, v in s.items()}
        got = _run(gs, x, rng.random(7).astype(np.float32), **par)
        keep = [0, 1, 2, 3, 5, 6]
        _check(x[keep], tuple(a[keep] for a in got), **{k: v[:6] for k, v in par.items()})
        assert got[0][4] == 11 and got[1][4] == 0 and got[2][4] == 1
    x[2] = torch.finfo(torch.float32).min      # all equal, all lowest: drawn evenly
    token, _, kept, _ = _run(gs, x[2:3], [0.5])
    assert token[0] == 500 and kept[0] == 1000


def test_uniform_out_of_range_and_nan_settings(gs):
    x = _logits(4, 500, 2, "fp16")
    got = _run(gs, x, [-1.0, 1.0, 7.0, float("nan")])
    _check(x, got)
    nan = float("nan")
    got = _run(gs, x, [0.3] * 4, temperature=[nan] * 4)
    _check(x, got, temperature=[0.0] * 4)
    got = _run(gs, x, [0.3] * 4, top_p=[nan] * 4, min_p=[nan] * 4, top_k=[-3] * 4)
    _check(x, got)


def test_frequencies(gs):
    """Draws over evenly spaced uniforms hit every token in proportion to its
    share of the kept prefix: counts are exact to one."""
    vocab, n = 64, 20000
    g = torch.Generator(device=DEV).manual_seed(9)
    row = torch.randn(vocab, device=DEV, generator=g)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    token, _, kept, _ = _run(gs, row.expand(n, vocab).contiguous(), u, top_p=[0.8] * n)
    s = row.cpu().double().numpy()
    order = np.argsort(-s)
    p = np.exp(s[order]) / np.exp(s).sum()
    k = int(np.searchsorted(np.cumsum(p), 0.8)) + 1
    assert (kept == k).all()
    want = p[:k] / p[:k].sum() * n
    count = np.bincount(token, minlength=vocab)[order[:k]]
    assert count.sum() == n and np.abs(count - want).max() <= 1.1


def test_stream_and_repeat(gs):
    """Another stream, and a second call: the same draws."""
    x = _logits(33, 59392, 8, "fp16")
    u = np.random.default_rng(1).random(33).astype(np.float32)
    par = dict(top_p=[0.95] * 33, temperature=[1.2] * 33)
    a = _run(gs, x, u, **par)
    b = _run(gs, x, u, stream=torch.cuda.Stream(), **par)
    assert all(np.array_equal(i, j) for i, j in zip(a, b))
    # one row alone (a wider cluster) draws what it draws in the batch
    one = _run(gs, x[7:8], u[7:8], top_p=[0.95], temperature=[1.2])
    assert one[0][0] == a[0][7] and one[1][0] == a[1][7] and one[2][0] == a[2][7]
