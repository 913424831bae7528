"""Checks of best_of_n.py that need no GPU: what is refused before any device
work."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


def _refused(bn, f, *args, **kw):
    with pytest.raises(bn.gs.GsError) as e:
        f(*args, **kw)
    assert e.value.code == bn.gs.GS_ERR_INVALID_ARG


def test_token_ids(bn):
    for good in ([0], [99, 0], np.array([5, 99]), torch.tensor([1, 2], dtype=torch.int32)):
        bn.check_tokens(good, 100)
    for bad in ([100], [-1], [3, 2 ** 40], np.array([0, 100]), torch.tensor([-5]), [1.0], [[1]],
                torch.tensor(3)):
        _refused(bn, bn.check_tokens, bad, 100)


def test_runs(bn):
    """Runs of one call name each place at most once."""
    for good, rows in (([(0, 0, [1, 2, 3])], 3), ([(0, 0, [1]), (1, 0, [1])], 2),
                       ([(0, 5, [1, 2]), (1, 3, [4]), (0, 7, [3, 4])], 5),
                       ([(0, 7, [3, 4]), (0, 5, [1, 2])], 4)):
        assert bn.check_runs(good, 5) == rows
    for bad in ([], [(0, 0, [])], [(0, 0, [1]), (1, 0, [])], [(0, 0, [1] * 6)],
                [(0, 0, [1, 2, 3]), (0, 2, [1])], [(0, 2, [1]), (1, 2, [1]), (0, 0, [1, 2, 3])],
                [(0, 4, [1]), (0, 4, [1])]):
        _refused(bn, bn.check_runs, bad, 5)


def test_uniforms(bn):
    """Any layout and type of the right shape becomes contiguous fp32 on the device."""
    g = torch.Generator().manual_seed(0)
    u = torch.rand(3, 5, generator=g)
    for given in (u, u.double(), u.t().contiguous().t(), torch.cat([u, u], 1)[:, :5], u.numpy(),
                  u.tolist()):
        got = bn.uniform_table(given, 3, 5, torch.device("cpu"))
        assert got.dtype == torch.float32 and got.is_contiguous() and torch.equal(got, u)
    assert bn.uniform_table(torch.empty(0, 5), 0, 5, torch.device("cpu")).shape == (0, 5)
    for bad in (u.t(), u[:2], u[:, :4], u[0], u[None], torch.tensor(0.5)):
        _refused(bn, bn.uniform_table, bad, 3, 5, torch.device("cpu"))
