"""gs_qlinear with more than 32 rows and many groups: places of tensor memory used over and
over, alone and with two calls at once.  Tolerances as in test_gpu_qlinear."""
import pytest
import torch

from tests.test_gpu_qlinear import DEV, TYPES, _check, _run, _weights, _x

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_many_stages(gs, dtype, group):
    """32 stages of 128 k in a slice, and 64 in one of few rows."""
    for N, K in ((8192, 8192), (130, 65536)):
        w, W = _weights(gs, dtype, N, K, group, True, False, seed=group, scale=0.02)
        x = _x(dtype, 544, K, seed=3)
        for M in (33, 128, 544):
            y, err = _run(gs, w, x[:M])
            assert err == 0
            _check(dtype, y, W, x[:M], w)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_two_calls_at_once(gs, group):
    """Two streams, each call's bits those of the call alone, every time."""
    w, _ = _weights(gs, "bf16", 8192, 8192, group, True, False, seed=group, scale=0.02)
    g, _ = _weights(gs, "bf16", 8192, 1024, group, False, True, seed=1, scale=0.02)
    xs = [_x("bf16", 300, 8192, seed=1), _x("bf16", 300, 1024, seed=2)]
    calls = ((w, xs[0], 8192, 0), (g, xs[1], 4096, 2))
    for rows in (33, 300):
        want = [_run(gs, m, x[:rows], epilogue=epi)[0] for m, x, _, epi in calls]
        outs = [torch.zeros(20, rows, n, dtype=TYPES["bf16"], device=DEV) for _, _, n, _ in calls]
        errs = torch.zeros(2, dtype=torch.int32, device=DEV)
        streams = [torch.cuda.Stream() for _ in calls]
        torch.cuda.synchronize()
        for i in range(20):
            for j, (m, x, n, epi) in enumerate(calls):
                gs.gs_qlinear(m, x.data_ptr(), x.stride(0), outs[j][i].data_ptr(), n, rows, epi,
                              errs[j:].data_ptr(), streams[j].cuda_stream)
        torch.cuda.synchronize()
        assert (errs == 0).all()
        for got, y in zip(outs, want):
            assert (got == y).all()
