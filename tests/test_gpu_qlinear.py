"""gs_qlinear against products in 64 bits.

Tolerances.  The kernel adds q x (in bf16 (16 + q) x) and takes the zero's part off
as a multiple of the sum of x.  With B = sum_k c s |x_k|, c = 15 in fp16 and 31 in
bf16, every partial sum is at most B.  A tensor instruction adds 16 products with an
error of at most 2^-22 of the sum so far: K / 16 of them; then come a sum of x, two
products and two sums per group, a sum per slice: (K / 8 + 32) 2^-23 B.  Then the
output's rounding, u |y| with u = 2^-11 (fp16) or 2^-8 (bf16), or 2^-24 (|y| + |acc|)
for fp32.  A gate's error passes through silu with a slope of at most 1.1, and its
exponential and quotient add 2^-20 of the result.

That bound is for the worst signs.  For random ones the sums' errors are far below the
output's rounding, which is evenly spread over at most u |y|: over many outputs the
mean square of the error is at most (u |y|)^2 / 3, of which 0.6 u leaves 4 per cent for
the rest."""
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


def _weights(gs, dtype, N, K, group, zeros, gated, seed=0, scale=0.05, stream=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randint(0, 16, (N, K), device=DEV, generator=g, dtype=torch.uint8)
    s = (scale * (0.5 + torch.rand(N, K // group, device=DEV, generator=g))).to(TYPES[dtype])
    z = torch.randint(0, 16, (N, K // group), device=DEV, generator=g, dtype=torch.uint8) if zeros else None
    w = gs.gs_qweight(0, N, K, group, gs.GS_F16 if dtype == "fp16" else gs.GS_BF16, int(zeros), int(gated))
    packed = torch.full((gs.gs_qweight_bytes(w) + 64,), 0x7F, dtype=torch.uint8, device=DEV)
    w.packed = packed.data_ptr()
    plain = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
    torch.cuda.synchronize()
    gs.gs_qweight_pack(w, plain.data_ptr(), s.data_ptr(), z.data_ptr() if zeros else 0,
                       (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    assert (packed[-64:] == 0x7F).all()
    w.held = packed                      # the descriptor names the memory, it does not own it
    w.sums = 15.0 if dtype == "fp16" else 31.0
    w.scales = s.double().repeat_interleave(group, 1)
    zz = 8 if z is None else z.double().repeat_interleave(group, 1)
    return w, (q.double() - zz) * s.double().repeat_interleave(group, 1)


def _run(gs, w, x, epilogue=0, y=None, ld=None, stream=None):
    outs = w.N // 2 if w.gated else w.N
    if y is None:
        y = torch.full((x.shape[0], ld or outs), 7.0, dtype=torch.float32 if epilogue == 1 else x.dtype,
                       device=DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    gs.gs_qlinear(w, x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), x.shape[0], epilogue,
                  err.data_ptr(), (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return y, int(err.item())


def _x(dtype, M, K, seed=1, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(M, K, device=DEV, generator=g)).to(TYPES[dtype])


def _bounds(w, x):
    return (w.K / 8 + 32) * 2.0 ** -23 * w.sums * (x.double().abs() @ w.scales.t())


def _check(dtype, y, W, x, w, gated=False):
    u = UNIT[dtype]
    acc, err = x.double() @ W.t(), _bounds(w, x)
    if gated:
        half = W.shape[0] // 2
        (ga, up), (eg, eu) = (t.split(half, dim=1) for t in (acc, err))
        silu = ga * torch.sigmoid(ga)
        acc = silu * up
        err = 1.1 * eg * (up.abs() + eu) + silu.abs() * eu + 2.0 ** -20 * acc.abs()
    bound = err + u * (acc.abs() + err) + 2.0 ** -25
    off = (y.double() - acc).abs()
    assert (off / bound).max().item() <= 1.0
    if acc.numel() >= 1000:
        assert off.square().mean().sqrt() <= 0.6 * u * acc.square().mean().sqrt()


SHAPES = [(1, 32), (7, 32), (16, 64), (40, 96), (128, 128), (129, 160), (1000, 1024), (130, 2080),
          (2048, 512), (264, 4096), (5000, 320)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
def test_shapes(gs, dtype, group, zeros):
    for i, (N, K) in enumerate(SHAPES):
        K = -(-K // group) * group
        w, W = _weights(gs, dtype, N, K, group, zeros, False, seed=i)
        for M in (1, 2, 8, 9, 17, 33, 129):
            x = _x(dtype, M, K, seed=M)
            y, err = _run(gs, w, x)
            assert err == 0
            _check(dtype, y, W, x, w)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("F,K,group", [(1, 32, 32), (8, 64, 64), (13, 96, 32), (64, 256, 128),
                                       (1000, 1024, 64), (4096, 1024, 32)])
def test_gated(gs, dtype, F, K, group):
    w, W = _weights(gs, dtype, 2 * F, K, group, True, True, seed=F, scale=0.02)
    for M in (1, 5, 16, 40, 130):
        x = _x(dtype, M, K, seed=M)
        y, err = _run(gs, w, x, epilogue=2)
        assert err == 0
        _check(dtype, y, W, x, w, gated=True)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_residual(gs, dtype):
    for N, K in ((7, 64), (1024, 1024), (515, 192)):
        w, W = _weights(gs, dtype, N, K, 64, True, False)
        for M in (1, 19, 70):
            x = _x(dtype, M, K)
            before = torch.randn(M, N + 3, device=DEV)
            y, err = _run(gs, w, x, epilogue=1, y=before.clone())
            assert err == 0 and torch.equal(y[:, N:], before[:, N:])
            acc, e = x.double() @ W.t(), _bounds(w, x)
            want = before[:, :N].double() + acc
            bound = e + 2.0 ** -24 * (want.abs() + acc.abs() + 2 * e) + 2.0 ** -30
            assert ((y[:, :N].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("N,K,gated", [(1024, 1024, False), (264, 4096, False), (2048, 640, True),
                                       (20000, 256, False)])
def test_rows_do_not_depend_on_the_batch(gs, dtype, N, K, gated):
    """A row has the same bits alone and in any batch of up to 32, and in any larger one, at any
    place of it."""
    w, W = _weights(gs, dtype, N, K, 64, True, gated, scale=0.02)
    x = _x(dtype, 300, K)
    epi = 2 if gated else 0
    many, err = _run(gs, w, x, epilogue=epi)
    assert err == 0
    few = torch.cat([_run(gs, w, x[a: a + 32], epilogue=epi)[0] for a in range(0, 300, 32)])
    for y in (many, few):
        _check(dtype, y, W, x, w, gated)
    for a, b in ((0, 1), (3, 4), (77, 78), (5, 13), (20, 36), (64, 96), (290, 299)):
        y, _ = _run(gs, w, x[a:b], epilogue=epi)
        assert torch.equal(y, few[a:b]), (a, b)
    for a, b in ((0, 33), (100, 150), (1, 66), (20, 148), (5, 134), (33, 290)):
        y, _ = _run(gs, w, x[a:b], epilogue=epi)
        assert torch.equal(y, many[a:b]), (a, b)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("N,K,group,zeros,gated", [
    (39991, 1024, 128, True, False), (24573, 2048, 64, False, False), (60000, 512, 32, True, False),
    (40002, 1024, 32, True, True), (19473, 512, 128, False, False)])
def test_many_outputs(gs, dtype, N, K, group, zeros, gated):
    """More tiles than a wave of blocks has warps: what goes on from tile to tile, the last tile
    cut short, what lies behind it left alone."""
    w, W = _weights(gs, dtype, N, K, group, zeros, gated, scale=0.02)
    epi, outs = 2 if gated else 0, N // 2 if gated else N
    x = _x(dtype, 130, K)
    many, err = _run(gs, w, x, epilogue=epi, ld=outs + 3)
    assert err == 0 and (many[:, outs:] == 7).all()
    _check(dtype, many[:, :outs], W, x, w, gated)
    x = x[:32]
    whole, err = _run(gs, w, x, epilogue=epi)
    assert err == 0
    _check(dtype, whole, W, x, w, gated)
    for a, b in ((0, 1), (3, 8), (8, 16), (9, 25), (15, 32)):
        y, err = _run(gs, w, x[a:b], epilogue=epi, ld=outs + 5)
        assert err == 0 and torch.equal(y[:, :outs], whole[a:b]) and (y[:, outs:] == 7).all(), (a, b)


def test_strides_and_streams(gs):
    """Rows apart in memory, odd output strides, what lies between is left alone."""
    for dtype in TYPES:
        w, W = _weights(gs, dtype, 200, 192, 64, True, False, stream=torch.cuda.Stream())
        wide = torch.full((21, 192 + 24), float("nan"), dtype=TYPES[dtype], device=DEV)
        wide[:, :192] = _x(dtype, 21, 192)
        plain, _ = _run(gs, w, wide[:, :192].contiguous())
        for ld in (200, 201, 202, 204, 333):
            y, err = _run(gs, w, wide[:, :192], ld=ld, stream=torch.cuda.Stream())
            assert err == 0 and torch.equal(y[:, :200], plain) and (y[:, 200:] == 7).all()
        wide = torch.full((70, 192 + 24), float("nan"), dtype=TYPES[dtype], device=DEV)
        wide[:, :192] = _x(dtype, 70, 192)
        many, _ = _run(gs, w, wide[:, :192].contiguous())
        for ld in (200, 201, 333):
            y, err = _run(gs, w, wide[:, :192], ld=ld, stream=torch.cuda.Stream())
            assert err == 0 and torch.equal(y[:, :200], many) and (y[:, 200:] == 7).all()
        wide = wide[:21]
        # an output that starts in the middle of eight bytes
        room = torch.full((21 * 300,), 7.0, dtype=TYPES[dtype], device=DEV)
        y, err = _run(gs, w, wide[:, :192], y=room[1: 1 + 21 * 204].view(21, 204))
        assert torch.equal(y[:, :200], plain) and (room[1 + 21 * 204:] == 7).all() and room[0] == 7


def test_values_that_are_not_finite(gs):
    """A row's infinities and NaN stay in that row."""
    w, _ = _weights(gs, "bf16", 300, 256, 32, True, False)
    for M in (12, 45):
        x = _x("bf16", M, 256)
        base, _ = _run(gs, w, x)
        x[3, 17], x[5, 200] = float("inf"), float("nan")
        y, _ = _run(gs, w, x)
        keep = [i for i in range(M) if i not in (3, 5)]
        assert torch.equal(y[keep], base[keep])
        # (an infinity times a weight of zero is NaN, times another one infinite)
        assert not torch.isfinite(y[3]).any() and torch.isnan(y[5]).all()


def test_range_word(gs):
    """An fp16 output beyond the type's range is infinite and raises the word."""
    w, W = _weights(gs, "fp16", 64, 128, 64, False, False, scale=40.0)
    x = _x("fp16", 3, 128, scale=100.0)
    x[1] = 0
    y, err = _run(gs, w, x)
    assert err == 3 and torch.isinf(y[0]).any() and (y[1] == 0).all()
    w, W = _weights(gs, "bf16", 64, 128, 64, False, False, scale=40.0)
    y, err = _run(gs, w, x.bfloat16())
    assert err == 0 and torch.isfinite(y).all()


def test_offsets_past_32_bits(gs):
    """Rows of inputs and outputs that lie more than 2^31 elements apart."""
    w, W = _weights(gs, "bf16", 48, 64, 32, False, False)
    far = 2 ** 31 + 64
    room = torch.zeros(far + 1024, dtype=torch.bfloat16, device=DEV)
    x = room.as_strided((2, 64), (far, 1))
    x.copy_(_x("bf16", 2, 64))
    out = torch.zeros(far + 1024, dtype=torch.bfloat16, device=DEV)
    y, err = _run(gs, w, x, y=out.as_strided((2, 48), (far, 1)))
    assert err == 0
    _check("bf16", y, W, x, w)
    far = 2 ** 26 + 8                    # (its row 32 lies beyond 2^31 elements)
    x = room.as_strided((33, 64), (far, 1))
    x.copy_(_x("bf16", 33, 64))
    y, err = _run(gs, w, x, y=out.as_strided((33, 48), (far, 1)))
    assert err == 0
    _check("bf16", y, W, x, w)


def test_captured_and_replayed(gs):
    w, W = _weights(gs, "fp16", 2048, 1024, 64, True, True, scale=0.02)
    for M in (17, 150):
        x, y = _x("fp16", M, 1024), torch.zeros(M, 1024, dtype=torch.float16, device=DEV)
        err = torch.zeros(1, dtype=torch.int32, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            gs.gs_qlinear(w, x.data_ptr(), 1024, y.data_ptr(), 1024, M, 2, err.data_ptr(),
                          torch.cuda.current_stream().cuda_stream)
        for seed in (1, 2):
            x.copy_(_x("fp16", M, 1024, seed=seed))
            graph.replay()
            torch.cuda.synchronize()
            want, _ = _run(gs, w, x, epilogue=2)
            assert torch.equal(y, want)
