"""gs_sample on rows whose logits depend on the token's index: rising, falling,
a likely stretch at either end, and half of the vocabulary at -inf.  The level
that divides a row is sampled at its start (each slice's), so these are the
rows on which it lies far off.  Checked like test_gpu_sample.py; and a draw from
a row of distinct logits does not depend on their places: its token is the one
that a shuffled row's draw has, at its own place."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import DEV, _check, _logits, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


SETTINGS = [dict(), dict(top_p=0.9), dict(top_p=0.999), dict(top_k=50), dict(top_k=6000),
            dict(min_p=0.05), dict(temperature=1.4, top_k=700, top_p=0.8, min_p=0.001)]


def _orders(x):
    """Permutations of each row's places: (name, indices [rows, vocab])."""
    rows, vocab = x.shape
    up = torch.argsort(x.float(), dim=-1, stable=True)
    yield "rising", up
    yield "falling", up.flip(-1)
    few = vocab // 10                           # the likely tenth, shuffled, ahead or behind
    g = torch.Generator(device=x.device).manual_seed(1)
    mix = torch.randperm(few, device=x.device, generator=g)
    yield "likely first", torch.cat([up.flip(-1)[:, :few][:, mix], up[:, : vocab - few]], 1)
    yield "likely last", torch.cat([up[:, : vocab - few], up.flip(-1)[:, :few][:, mix]], 1)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows", [7, 20, 40, 90])
def test_orders(gs, dtype, rows):
    """Clusters of eight, four and two blocks for a row, and one block."""
    vocab = 59392
    x = _logits(rows, vocab, rows, dtype)
    rng = np.random.default_rng(rows)
    for s in SETTINGS:
        par = {k: [v] * rows for k, v in s.items()}
        u = rng.random(rows).astype(np.float32)
        for _, at in _orders(x):
            y = x.gather(1, at)
            _check(y, _run(gs, y, u, **par), **par)


@pytest.mark.parametrize("rows", [7, 20, 40, 90])
def test_places_do_not_matter(gs, rows):
    """Distinct logits: the same draw wherever they stand, to the bit."""
    vocab = 40001
    v = (-1.3 * torch.log1p(torch.arange(vocab, dtype=torch.float64))).float().to(DEV)
    assert (v.diff() < 0).all()
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.stack([v[torch.randperm(vocab, device=DEV, generator=g)] for _ in range(rows)])
    u = np.random.default_rng(rows).random(rows).astype(np.float32)
    for s in SETTINGS:
        par = {k: [v] * rows for k, v in s.items()}
        token, logprob, kept, _ = _run(gs, x, u, **par)
        for name, at in _orders(x):
            t2, l2, k2, _ = _run(gs, x.gather(1, at), u, **par)
            there = at.cpu().numpy()[np.arange(rows), t2]
            assert np.array_equal(there, token), name
            assert np.array_equal(l2, logprob) and np.array_equal(k2, kept), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [7, 20, 40, 90])
def test_half_of_the_vocabulary_masked(gs, dtype, rows):
    """-inf in the first half, the second, one slice, all but a few, every other token."""
    vocab = 59392
    x = _logits(rows, vocab, rows + 1, dtype)
    rng = np.random.default_rng(rows)
    i = torch.arange(vocab, device=DEV)
    for mask in (i < vocab // 2, i >= vocab // 2, (i >= vocab // 8) & (i < vocab // 4),
                 (i < vocab // 3) | (i > vocab // 3 + 30), i % 2 == 0):
        y = x.masked_fill(mask, float("-inf"))
        for s in SETTINGS:
            par = {k: [v] * rows for k, v in s.items()}
            _check(y, _run(gs, y, rng.random(rows).astype(np.float32), **par), **par)
