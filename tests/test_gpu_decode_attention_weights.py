"""gs_decode_attention where one key outweighs all others by far.

The tolerance is the one of test_gpu_decode_attention.py: 2.1 u A + 1e-4 A with
A = sum_j p_j |v_j|, u the unit of the cache's type, and half of fp16's
smallest subnormal for the output's own rounding.  It is relative to what the
values contribute, so a small weight must carry the type's relative precision
like a large one: the heaviest key's value is 0 here, and all of A comes from
the light keys.  A score is one product (one dim is not zero).  The weights go
down to 2^-29, where 2^15 times them is fp16's smallest normal."""
import pytest
import torch

from tests.test_gpu_decode_attention import DEV, _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1)])
@pytest.mark.parametrize("below", [2.0, 9.0, 12.0, 16.0, 17.5, 18.0, 20.0])
def test_light_keys_beside_a_heavy_one(gs, dtype, D, Hq, Hkv, below):
    """exp(-below) for every key but one: the first, or one in the middle."""
    ns = [2, 33, 64, 700, 2100]
    c = _case(dtype, ns, Hq, Hkv, D, seed=3)
    t = c["table"].cpu()
    c["q"].zero_()
    c["q"][:, :, 5] = 8.0
    step = below * D ** 0.5 / 8.0                            # scale is D^-0.5
    K, V = (c["pool"].view(-1, 2, Hkv, *s) for s in ((64, D), (D, 64)))
    for b, n in enumerate(ns):
        heavy = 0 if b % 2 == 0 else n // 2
        k = torch.zeros(n, Hkv, D, dtype=c["q"].dtype, device=DEV)
        k[:, :, 5] = -step
        k[heavy] = 0
        v = c["v"][b].abs() * 1000
        v[heavy] = 0
        c["k"][b], c["v"][b] = k, v
        at = torch.arange(n, device=DEV)
        pg = t[b].to(DEV)[at // 64].long()
        K[pg, 0, :, at % 64] = k
        V[pg, 1, :, :, at % 64] = v
    for split in (0, 1, 1000):
        out, lse, err = _run(gs, c, split=split)
        assert err == 0
        _check(c, out, lse)
