"""StepDecoder.keep refuses choices whose numbers do not lie one behind another."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_choices_that_are_not_contiguous():
    from paper_2609_26638_gb300 import best_of_n as bn, gs
    shape = bn.Shape()
    dec = bn.StepDecoder(shape, bn.random_weights(shape), n_pages=3, max_seqs=2, max_ctx=128, max_rows=40)
    trees = [(dec.pool.open(), 0, [1, 2], [-1, 0])]
    dec.feed_trees(trees)
    apart = torch.zeros(1, 4, dtype=torch.int32, device=DEV)[:, ::2]
    assert apart.shape == (1, 2) and not apart.is_contiguous()
    with pytest.raises(gs.GsError) as e:
        dec.keep(trees, apart)
    assert e.value.code == gs.GS_ERR_INVALID_ARG
    more = [trees[0], (dec.pool.open(), 0, [3, 4], [-1, 0])]
    dec.feed_trees(more)
    crossed = torch.zeros(2, 2, dtype=torch.int32, device=DEV).t()
    with pytest.raises(gs.GsError):
        dec.keep(more, crossed)
    assert len(dec.keep(more, crossed.contiguous())) == 2
    dec.check()
