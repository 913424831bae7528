"""quantize at the ends of the types' ranges: each weight comes back within half a step (a
whole one with zeros, which are rounded themselves) and what a normal scale's rounding adds."""
import pytest
import torch


@pytest.fixture(scope="module")
def qweight():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import qweight
    return qweight


def _check(qweight, w, zeros):
    q, scale, zero = qweight.quantize(w, 32, zeros)
    assert torch.isfinite(scale).all()
    whole = torch.stack([q & 15, q >> 4], -1).flatten(1).double()
    z = 8.0 if zero is None else zero.double().repeat_interleave(32, 1)
    s = scale.double().repeat_interleave(32, 1)
    back = (whole - z) * s
    steps = (1.0 if zeros else 0.5) + 15 * torch.finfo(w.dtype).eps
    assert ((back - w.double()).abs() <= steps * s).all()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("size", [2.0 ** -24, 2.0 ** -23, 3e-7, 1e-6, 1e-5, 1e-3])
def test_small_weights(qweight, size, zeros):
    g = torch.Generator().manual_seed(1)
    for k in range(8):
        _check(qweight, (size * (1 + k / 8) * torch.randn(20, 128, generator=g)).half(), zeros)


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_largest_weights(qweight, dtype, zeros):
    w = torch.zeros(4, 64, dtype=dtype)
    most = torch.finfo(dtype).max
    w[0, 0], w[0, 1], w[1, 5], w[2, 7] = most, -most, most, -most
    _check(qweight, w, zeros)


@pytest.mark.parametrize("zeros", [False, True])
def test_strided_matrices(qweight, zeros):
    """A transposed matrix, and columns of a wider one, as their copies."""
    w = torch.randn(128, 96, generator=torch.Generator().manual_seed(3)).half()
    for view in (w.t(), w[:, :64], w.t()[::2, 32:96]):
        for a, b in zip(qweight.quantize(view, 64 if view.shape[1] % 64 == 0 else 32, zeros),
                        qweight.quantize(view.contiguous(), 64 if view.shape[1] % 64 == 0 else 32, zeros)):
            assert a is b is None or torch.equal(a, b) and a.is_contiguous()
