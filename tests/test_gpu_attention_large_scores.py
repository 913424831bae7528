"""The attentions over the paged cache with scores so large that fp32 is coarse there.

A score is 16 A B + U c: A from a row's own few bits, B a power of two, U the spacing of fp32 at
the score's size 2^x, and c whole numbers that rise from page to page by some units of
log2.  Products and sums are multiples of U below 2^(x + 1), so every score is exact in fp32, in
whatever order it is summed, and so are differences of scores: what the definition in 64
bits says has to come out within the tolerance of small scores (test_gpu_tree_attention).
The log-sum-exp is the largest score times factors, four roundings of 2^-24 and that of fp32
itself: 2^-21 of it."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_tree_attention import DEV, TYPES, _cache, _case, _check, _dev, _run

pytestmark = pytest.mark.gpu
SIZES = [("fp16", x) for x in (20, 24, 25, 26, 27, 28, 30, 32, 34)] + [
    ("bf16", x) for x in (24, 27, 29, 30, 31, 34, 60, 100)]


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _large(c, x, rise):
    """The case with scores of 2^x .. 2^(x + 1) whose largest rises by about `rise` (log2 units)
    every 64 tokens, or by the spacing, if that is more."""
    D, Hkv = c["D"], c["Hkv"]
    unit = x - 23
    step = max(1, round(rise / (2.0 ** unit * D ** -0.5 * math.log2(math.e))))
    a = (x - 4) // 2
    q = torch.zeros(c["q"].shape, dtype=torch.float64, device=DEV)
    rows = torch.arange(q[..., 0].numel(), device=DEV).view(q.shape[:3])
    q[..., :16] = (2.0 ** a * (1 + rows % 32 / 32))[..., None]
    q[..., 16:18] = 2.0 ** unit
    c["q"] = q.to(TYPES[c["dtype"]])
    rng = np.random.default_rng(x)
    table = c["table"].cpu().numpy()
    for b, k in enumerate(c["k"]):
        t = np.arange(k.shape[0])
        lift = torch.from_numpy(t // 64 * step + rng.integers(0, step + 1, t.size)).to(DEV)
        assert t.size == 0 or int(lift.max()) < 128 * 128
        new = torch.zeros(k.shape, dtype=torch.float64, device=DEV)
        new[..., :16] = 2.0 ** (x - 4 - a)
        new[..., 16] = (lift % 128)[:, None]
        new[..., 17] = (lift - lift % 128)[:, None]
        c["k"][b] = new.to(TYPES[c["dtype"]])
        assert torch.equal(c["k"][b].double(), new)          # nothing is rounded on the way
        page = torch.from_numpy(table[b]).to(DEV)[torch.from_numpy(t // 64).to(DEV)]
        c["pool"].view(-1, 2, Hkv, 64, D)[page, 0, :, torch.from_numpy(t % 64).to(DEV)] = c["k"][b]
    assert torch.isfinite(c["q"]).all()
    return dict(slack=1e-4, lse_slack=1e-4 + 2.0 ** (x + 1) * D ** -0.5 * 2.0 ** -21)


@pytest.mark.parametrize("dtype,x", SIZES)
@pytest.mark.parametrize("D,nodes", [(64, 3), (128, 2), (64, 40), (128, 20)])
def test_trees(gs, dtype, x, D, nodes):
    for rise in (0, 4, 9, 12, 16):
        c = _case(dtype, [0, 5, 64, 700, 300], nodes, 8, 2, D, seed=x + rise)
        tol = _large(c, x, rise)
        for split in (0, 1, 4):
            out, lse, err = _run(gs, c, split=split)
            assert err == 0
            _check(c, out, lse, **tol)


@pytest.mark.parametrize("dtype,x", SIZES)
@pytest.mark.parametrize("D", [64, 128])
def test_single_tokens(gs, dtype, x, D):
    ns = [0, 5, 64, 700, 300]
    for rise in (0, 4, 9, 12, 16):
        c = _case(dtype, ns, 1, 8, 2, D, seed=x + rise)
        tol = _large(c, x, rise)
        cache = _cache(gs, c["pool"], c["table"], 2, D, dtype)
        n = _dev(np.array(ns) + 1)
        for split in (0, 1, 4):
            out = torch.zeros(5, 8 * D, dtype=TYPES[dtype], device=DEV)
            lse = torch.zeros(5, 8, device=DEV)
            scratch = torch.zeros(gs.gs_decode_attention_scratch_bytes(cache, 5, 8, split), dtype=torch.uint8,
                                  device=DEV)
            gs.gs_decode_attention(cache, c["q"].data_ptr(), 8 * D, 0, n.data_ptr(), 5, 8, D ** -0.5, 0,
                                   out.data_ptr(), 8 * D, lse.data_ptr(), split, scratch.data_ptr(),
                                   scratch.numel(), torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            assert int(scratch[:4].view(torch.int32).item()) == 0
            _check(c, out, lse, **tol)
