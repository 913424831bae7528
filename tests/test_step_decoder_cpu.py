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
