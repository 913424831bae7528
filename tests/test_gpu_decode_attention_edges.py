"""gs_decode_attention with scores at the ends of their range: keys of minus
infinity (whole steps, whole items, all keys but one, all keys), and scores of
several hundred.  Tolerances as in test_gpu_decode_attention.py; a key of minus
infinity has exactly no weight, so its value (large and finite) must not show."""
import pytest
import torch

from tests.test_gpu_decode_attention import DEV, UNIT, _case, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _rewrite(c, b):
    """Puts sequence b's keys and values into its pages anew."""
    n, Hkv, D = c["ns"][b], c["Hkv"], c["D"]
    at = torch.arange(n, device=DEV)
    pg = c["table"][b].long()[at // 64]
    c["pool"].view(-1, 2, Hkv, 64, D)[pg, 0, :, at % 64] = c["k"][b]
    c["pool"].view(-1, 2, Hkv, D, 64)[pg, 1, :, :, at % 64] = c["v"][b]


def _want(c, b):
    Hkv, D = c["Hkv"], c["D"]
    k, v = c["k"][b].double(), c["v"][b].double()
    s = torch.einsum("hgd,nhd->hgn", c["q"][b].double().view(Hkv, -1, D), k) * D ** -0.5
    return s, v


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 4), (12, 1)])
@pytest.mark.parametrize("split", [0, 2, 1000])
def test_keys_of_minus_infinity(gs, dtype, D, Hq, Hkv, split):
    ns = [700, 700, 700, 300, 300, 40]
    c = _case(dtype, ns, Hq, Hkv, D, seed=11)
    c["q"][:, :, 0] = c["q"][:, :, 0].abs() + 0.5          # (0 times infinity is NaN)
    none = [torch.zeros(n, dtype=torch.bool, device=DEV) for n in ns]
    none[0][32:64] = True                                    # one step of a warp
    none[0][640:] = True                                     # and the last, ragged ones
    none[1][128:256] = True                                  # an item of two pages
    none[1][:64] = True                                      # and the first page
    none[2][::3] = True                                      # here and there
    none[3][:-1] = True                                      # all but the last
    none[4][1:] = True                                       # all but the first
    none[5][:] = True                                        # all
    for b in range(len(ns)):
        c["k"][b][none[b], :, 0] = float("-inf")
        c["v"][b][none[b]] = 30000.0
        _rewrite(c, b)
    out, lse, err = _run(gs, c, split=split)
    assert err == 0
    u = UNIT[dtype]
    for b, n in enumerate(ns):
        o = out[b].double().view(Hkv, -1, D)
        if none[b].all():
            assert (o == 0).all() and (lse[b] == float("-inf")).all()
            continue
        s, v = _want(c, b)
        p = torch.softmax(s, -1)
        assert (p[:, :, none[b]] == 0).all()
        want = torch.einsum("hgn,nhd->hgd", p, v)
        bound = (2.1 * u + 1e-4) * torch.einsum("hgn,nhd->hgd", p, v.abs()) + 2.0 ** -24
        assert ((o - want).abs() <= bound).all(), (b, ((o - want).abs() / bound).max().item())
        assert (lse[b].double() - torch.logsumexp(s, -1).view(-1)).abs().max() <= 5e-5
        if int((~none[b]).sum()) == 1:                       # one key left: its value, exactly
            only = c["v"][b][~none[b]][0].view(Hkv, 1, D).expand(Hkv, Hq // Hkv, D)
            assert torch.equal(out[b].view(Hkv, -1, D), only)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_several_hundred(gs, dtype, D):
    """Queries and keys of one sign: scores from about 350 to 850, of both signs.

    A score is a sum of D fp32 products, all of one sign and below 2048 / sqrt(D)
    in all before scaling: its error is at most D 2^-24 of it, and three more
    roundings (scale, maximum, exponent's argument) of 2^-24 each: for |s| up to
    1000, 1000 (D + 3) 2^-24 = 0.008 at most, and twice that for a ratio of two
    weights; lse is off by at most 0.008 and its own rounding, 1000 2^-24."""
    ns = [900, 65, 3]
    c = _case(dtype, ns, 8, 2, D, seed=12)
    c["q"] = c["q"].abs() * 3.0
    worst = 0.0
    for sign in (1.0, -1.0):
        for b, n in enumerate(ns):
            g = torch.Generator(device=DEV).manual_seed(b)
            k = torch.rand(n, 2, D, device=DEV, generator=g) * 2 + 14.0
            c["k"][b] = (sign * k * (64 / D) ** 0.5).to(c["q"].dtype)
            _rewrite(c, b)
        for split in (0, 1):
            out, lse, err = _run(gs, c, split=split)
            assert err == 0
            for b, n in enumerate(ns):
                s, v = _want(c, b)
                worst = max(worst, s.abs().max().item())
                e = 1000 * (D + 3) * 2.0 ** -24
                p = torch.softmax(s, -1)
                want = torch.einsum("hgn,nhd->hgd", p, v)
                mass = torch.einsum("hgn,nhd->hgd", p, v.abs())
                bound = (2.1 * UNIT[dtype] + 2 * e) * mass + 2.0 ** -24
                assert ((out[b].double().view(2, -1, D) - want).abs() <= bound).all()
                assert (lse[b].double() - torch.logsumexp(s, -1).view(-1)).abs().max() <= e + 6e-5
    assert 300 < worst < 1000
