"""gs_decode_attention over page tables far wider than the rows are long, as a
pool of a large capacity has them, with the split left open.  The table's unused
entries are no page numbers: one that is read raises the error word.
Tolerances and checks of test_gpu_decode_attention.py."""
import pytest
import torch

from tests.test_gpu_decode_attention import DEV, _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _widen(c, per):
    t = c["table"]
    c["table"] = torch.cat([t, torch.full((t.shape[0], per - t.shape[1]), 2 ** 30, dtype=torch.int32,
                                          device=DEV)], 1).contiguous()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("per", [60, 512, 2048, 20000])
@pytest.mark.parametrize("ns", [[517], [3000], [0], [1, 517], [0, 64, 129, 2000] * 8, [400] * 64])
def test_wide_table(gs, D, per, ns):
    c = _case("bf16", ns, 8, 4, D, seed=len(ns) + D)
    _widen(c, per)
    for window in (0, 100):
        out, lse, err = _run(gs, c, window=window)
        assert err == 0
        _check(c, out, lse, window)


def test_entries_are_read_up_to_the_length_alone(gs):
    """The entry of a row's last page is read, the one behind it is not."""
    c = _case("fp16", [64 * 7, 64 * 7 + 1], 8, 4, 64, seed=1)
    c["table"][0, 7] = -1
    _widen(c, 900)
    out, lse, err = _run(gs, c)
    assert err == 0
    _check(c, out, lse)
    c["table"][1, 7] = 2 ** 30
    assert _run(gs, c)[2] == 1
