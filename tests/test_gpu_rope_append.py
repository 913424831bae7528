"""gs_rope_table and gs_rope_append against the definition in 64 bits.

Tolerances: the operator works in fp32 and rounds each output once, so an
output is within half a unit of its type (2^-11 of the value in fp16, 2^-8 in
bf16, and the smallest fp16 subnormal's half) of a value that carries the fp32
arithmetic's error: about 10 roundings of 2^-24, and of the sum over the head,
taken here as 1e-5 of the head's largest value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
HALF_UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _table(gs, rot, rows, theta=10000.0, **kw):
    t = torch.full((rows, rot // 2, 2), float("nan"), device=DEV)
    sc = gs.gs_rope_scaling(kind=kw.pop("kind", gs.ROPE_PLAIN), theta=theta, **kw)
    gs.gs_rope_table(sc, rot, rows, t.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return t


def _want_frequencies(gs, rot, theta, kind, factor, ctx=0, fast=0.0, slow=0.0):
    i = np.arange(rot // 2)
    if kind == gs.ROPE_NTK:
        theta = theta * factor ** (rot / (rot - 2))
    inv = theta ** (-2.0 * i / rot)
    if kind == gs.ROPE_LINEAR:
        inv = inv / factor
    if kind == gs.ROPE_YARN:
        def pair(turns):
            return rot * np.log(ctx / (turns * 2 * np.pi)) / (2 * np.log(theta))
        lo, hi = max(np.floor(pair(fast)), 0), min(np.ceil(pair(slow)), rot - 1)
        ramp = np.clip((i - lo) / max(hi - lo, 1e-3), 0, 1)
        inv = inv * (1 - ramp) + inv / factor * ramp
    return inv


@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("kind", ["PLAIN", "LINEAR", "NTK", "YARN"])
def test_table(gs, rot, kind):
    k = getattr(gs, "ROPE_" + kind)
    rows = 70001
    kw = dict(factor=4.0, original_ctx=16384, beta_fast=32.0, beta_slow=1.0)
    got = _table(gs, rot, rows, 500000.0, kind=k, **kw).cpu().double().numpy()
    at = np.array([0, 1, 2, 63, 4097, 65535, 70000])
    angle = at[:, None] * _want_frequencies(gs, rot, 500000.0, k, 4.0, 16384, 32.0, 1.0)[None]
    mag = 0.1 * np.log(4.0) + 1 if kind == "YARN" else 1.0
    # one rounding to fp32 (2^-25 of at most 1.14), and the 64-bit angle's own error
    np.testing.assert_allclose(got[at, :, 0], mag * np.cos(angle), atol=8e-8, rtol=0)
    np.testing.assert_allclose(got[at, :, 1], mag * np.sin(angle), atol=8e-8, rtol=0)


def _place(tokens, seqs, first, rng):
    """Runs of tokens per sequence at their own first slot."""
    seq = np.sort(rng.integers(0, seqs, tokens)) if tokens != seqs else np.arange(tokens)
    slot = np.empty(tokens, np.int64)
    for s in range(seqs):
        w = np.flatnonzero(seq == s)
        slot[w] = first + 5 * s + np.arange(len(w))
    return seq, slot


def _case(dtype, T, seqs, first, Hq, Hkv, D, seed, pad=0):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    seq, slot = _place(T, seqs, first, rng)
    per = int(slot.max()) // 64 + 1
    n_pages = seqs * per + 2
    table = rng.permutation(n_pages)[: seqs * per].reshape(seqs, per)
    width = (Hq + 2 * Hkv) * D
    qkv = torch.randn(T, width + pad, device=DEV, generator=g).to(TYPES[dtype])
    pool = torch.randn(n_pages, 2, Hkv, 64 * D, device=DEV, generator=g).to(TYPES[dtype])
    gains = [(1 + 0.2 * torch.randn(D, device=DEV, generator=g)).bfloat16() for _ in range(2)]
    pos = slot + rng.integers(0, 7, T)
    return dict(seq=seq, slot=slot, pos=pos, table=table, qkv=qkv, pool=pool, gains=gains, D=D,
                Hq=Hq, Hkv=Hkv, dtype=dtype, T=T)


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _run(gs, c, rope, norm, q=None, stream=None):
    ids = [_i32(c[k]) for k in ("seq", "slot", "pos")]
    table = _i32(c["table"])
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.zeros(c["T"], c["Hq"] * c["D"], dtype=c["qkv"].dtype, device=DEV) if q is None else q
    cache = gs.gs_cache(c["pool"].data_ptr(), c["pool"].shape[0], c["Hkv"], c["D"],
                        gs.GS_F16 if c["dtype"] == "fp16" else gs.GS_BF16, table.data_ptr(),
                        table.shape[0], table.shape[1])
    qg, kg = (c["gains"][0].data_ptr(), c["gains"][1].data_ptr()) if norm else (0, 0)
    torch.cuda.synchronize()
    gs.gs_rope_append(cache, rope, c["qkv"].data_ptr(), c["qkv"].stride(0), c["T"], c["Hq"], qg, kg,
                      1e-6, ids[0].data_ptr(), ids[1].data_ptr(), ids[2].data_ptr(), q.data_ptr(),
                      q.stride(0), err.data_ptr(),
                      (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return q, int(err.item())


def _want(c, angles, half, norm, rot):
    Hq, Hkv, D, T = c["Hq"], c["Hkv"], c["D"], c["T"]
    x = c["qkv"][:, : (Hq + 2 * Hkv) * D].cpu().double().numpy().reshape(T, Hq + 2 * Hkv, D)
    y = x[:, : Hq + Hkv].copy()
    if norm:
        y /= np.sqrt((y ** 2).mean(-1, keepdims=True) + 1e-6)
        y[:, :Hq] *= c["gains"][0].cpu().double().numpy()
        y[:, Hq:] *= c["gains"][1].cpu().double().numpy()
    a = angles[c["pos"]][:, None]
    i = np.arange(rot // 2)
    f, s = (i, i + rot // 2) if half else (2 * i, 2 * i + 1)
    p, q = y[..., f].copy(), y[..., s].copy()
    y[..., f] = p * np.cos(a) - q * np.sin(a)
    y[..., s] = q * np.cos(a) + p * np.sin(a)
    return y[:, :Hq], y[:, Hq:], x[:, Hq + Hkv:]


def _close(got, want, dtype):
    bound = HALF_UNIT[dtype] * np.abs(want) + 1e-5 * np.abs(want).max(-1, keepdims=True) + 2.0 ** -25
    worst = (np.abs(got - want) / bound).max()
    assert worst <= 1.0, worst


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("T,seqs,first,Hq,Hkv,D,rot,half,norm", [
    (1, 1, 0, 4, 4, 64, 64, True, True),
    (1, 1, 63, 16, 8, 64, 32, False, True),
    (37, 37, 60, 16, 8, 64, 64, True, False),     # decode batch: single tokens
    (129, 1, 0, 8, 1, 128, 128, True, True),      # a prompt from slot 0
    (200, 1, 3, 12, 2, 64, 48, True, True),       # a prompt at an odd slot: runs cross tiles
    (333, 7, 61, 5, 5, 128, 16, False, True),     # several ragged runs
    (70, 3, 120, 32, 8, 128, 96, False, False),
])
def test_append(gs, dtype, T, seqs, first, Hq, Hkv, D, rot, half, norm):
    c = _case(dtype, T, seqs, first, Hq, Hkv, D, seed=T + rot)
    rows = int(c["pos"].max()) + 1
    table = _table(gs, rot, rows)
    before = c["pool"].clone()
    rope = gs.gs_rope(table.data_ptr(), rows, rot, gs.ROPE_HALF if half else gs.ROPE_INTERLEAVED)
    q, err = _run(gs, c, rope, norm)
    assert err == 0
    angles = np.arange(rows)[:, None] * (10000.0 ** (-2.0 * np.arange(rot // 2) / rot))[None]
    wq, wk, wv = _want(c, angles, half, norm, rot)
    _close(q.cpu().double().numpy().reshape(T, Hq, D), wq, dtype)
    page, at = c["table"][c["seq"], c["slot"] // 64], c["slot"] % 64
    K = c["pool"].view(-1, 2, Hkv, 64, D)
    V = c["pool"].view(-1, 2, Hkv, D, 64)
    pg, tk = torch.from_numpy(page).to(DEV), torch.from_numpy(at).to(DEV)
    _close(K[pg, 0, :, tk].cpu().double().numpy(), wk, dtype)
    assert np.array_equal(V[pg, 1, :, :, tk].cpu().double().numpy(), wv)    # values are copied
    # nothing else changed
    K[pg, 0, :, tk] = before.view(-1, 2, Hkv, 64, D)[pg, 0, :, tk]
    V[pg, 1, :, :, tk] = before.view(-1, 2, Hkv, D, 64)[pg, 1, :, :, tk]
    assert torch.equal(c["pool"].view(torch.int16), before.view(torch.int16))


def test_strides_in_place_and_streams(gs):
    """A row stride wider than the row; queries written over the projection's
    own; a stream other than the current one: the same bits."""
    c = _case("bf16", 45, 2, 17, 8, 2, 64, seed=9, pad=24)
    table = _table(gs, 64, 256)
    rope = gs.gs_rope(table.data_ptr(), 256, 64, gs.ROPE_HALF)
    pool0, qkv0 = c["pool"].clone(), c["qkv"].clone()
    q, _ = _run(gs, c, rope, True)
    pool1 = c["pool"].clone()
    c["pool"].copy_(pool0)
    side = torch.cuda.Stream()
    q2, _ = _run(gs, c, rope, True, stream=side)
    assert torch.equal(q, q2) and torch.equal(pool1, c["pool"])
    c["pool"].copy_(pool0)
    _run(gs, c, rope, True, q=c["qkv"])
    assert torch.equal(c["qkv"][:, : 8 * 64], q) and torch.equal(pool1, c["pool"])
    assert torch.equal(c["qkv"][:, 8 * 64:], qkv0[:, 8 * 64:])


def test_unwritten_tokens_and_error_word(gs):
    """Slot -1 writes nothing; indices out of range write nothing and raise the word."""
    table = _table(gs, 32, 512)
    rope = gs.gs_rope(table.data_ptr(), 512, 32, gs.ROPE_INTERLEAVED)
    for what in ("skip", "seq", "slot", "page", "pos"):
        c = _case("fp16", 9, 9, 5, 4, 2, 64, seed=3)
        c["pos"] = c["slot"].copy()
        if what == "skip":
            c["slot"][4] = -1
        elif what == "seq":
            c["seq"][4] = 9
        elif what == "slot":
            c["slot"][4] = c["table"].shape[1] * 64
        elif what == "page":
            c["table"][4] = c["pool"].shape[0]
        else:
            c["pos"][4] = 512
        before = c["pool"].clone()
        q, err = _run(gs, c, rope, True)
        assert err == (0 if what == "skip" else 1), what
        assert torch.isfinite(q).all()
        changed = (c["pool"].view(torch.int16) != before.view(torch.int16)).flatten(1).any(1)
        assert int(changed.sum()) == (9 if what == "pos" else 8), what


def test_head_of_zeros_and_large_values(gs):
    """A head of zeros stays zero; values whose squares pass fp16's range are normed in fp32."""
    c = _case("fp16", 3, 1, 0, 2, 2, 64, seed=1)
    c["qkv"][0] = 0
    c["qkv"][1] = 60000.0
    table = _table(gs, 64, 64)
    q, err = _run(gs, c, gs.gs_rope(table.data_ptr(), 64, 64, gs.ROPE_HALF), True)
    assert err == 0 and torch.isfinite(q).all() and (q[0] == 0).all()
    angles = np.arange(64)[:, None] * (10000.0 ** (-2.0 * np.arange(32) / 64))[None]
    _close(q.cpu().double().numpy().reshape(3, 2, 64), _want(c, angles, True, True, 64)[0], "fp16")
