"""gs_sample on rows with several logits of +inf: they share all the weight, and
a draw is one among them.  Everything is exact: with m infinite logits of which
top-k and then top-p keep z = ceil(p min(m, k)) (1 at least), the token is the
min(floor(u z), z - 1)-th of them by index, kept is z and logprob -ln z."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from tests.test_gpu_sample import TYPES, _logits, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _exact(where, u, top_k, top_p):
    m = len(where)
    if top_k > 0:
        m = min(m, top_k)
    if top_p < 1:
        m = max(math.ceil(Fraction(float(np.float32(top_p))) * m), 1)
    return where[min(math.floor(Fraction(float(np.float32(u))) * m), m - 1)], m


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 59392), (5, 59392), (200, 59392), (3, 131071), (2, 700)])
@pytest.mark.parametrize("count", [2, 37, 600])
def test_several_infinite_logits(gs, dtype, rows, vocab, count):
    """One block, and clusters whose blocks hold some or none of them each."""
    rng = np.random.default_rng(rows + vocab + count)
    x = _logits(rows, vocab, count, dtype)
    x[:, vocab // 3] = float("nan")
    where = []
    for r in range(rows):
        pool = np.setdiff1d(np.arange(vocab), [vocab // 3])
        if r % 3 == 1:                           # all in one stretch: other slices have none
            pool = pool[-min(2 * count, len(pool)):]
        w = np.sort(rng.choice(pool, min(count, len(pool)), replace=False))
        if r % 3 == 2:                           # the ends of the row among them
            w[0], w[-1] = 0, vocab - 1
        x[r, torch.from_numpy(w).to(x.device)] = float("inf")
        where.append(w)
    assert x.dtype == TYPES[dtype]
    for top_k in (0, 1, count - 1, count + 5):
        for top_p in (0.0, 0.5, 0.77, 1.0):
            u = rng.random(rows).astype(np.float32)
            u[0] = rng.choice(np.float32([0.0, 0.5, 0.99999994]))
            par = dict(top_k=[top_k] * rows, top_p=[top_p] * rows,
                       temperature=rng.choice([0.3, 1.0, 2.0], rows).tolist())
            token, logprob, kept, _ = _run(gs, x, u, **par)
            for r in range(rows):
                t, z = _exact(where[r], u[r], top_k, top_p)
                assert (token[r], kept[r]) == (t, z), (r, top_k, top_p, u[r])
                assert abs(logprob[r] + math.log(z)) <= 1e-6
    token, logprob, kept, _ = _run(gs, x, [0.9] * rows, temperature=[0.0] * rows)
    assert all(token[r] == where[r][0] for r in range(rows))
    assert (kept == 1).all() and (logprob == 0).all()
