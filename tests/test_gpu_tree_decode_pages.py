"""Decoding with drafted trees in pools that hold the texts and little or nothing more: drafts
take what room there is, and give it back."""
import numpy as np
import pytest

from tests.test_gpu_tree_decode import _greedy_or_near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


@pytest.fixture(scope="module")
def td():
    from paper_2609_26638_gb300 import tree_decode
    return tree_decode


def _pages(prompt, new):
    return -(-(len(prompt) + new - 1) // 64)              # the last token is not cached


def _wide(history, max_nodes, depth, ngram):
    """As many nodes as there may be, wrong but by luck."""
    return [history[-1]] + [(history[-1] + 1 + i) % 7 for i in range(max_nodes - 1)], [-1] + [0] * (max_nodes - 1)


@pytest.mark.parametrize("spare", [0, 1, 2])
@pytest.mark.parametrize("lengths,new", [((60, 60), 10), ((1, 63, 64, 130), 70), ((120,), 9)])
def test_pools_of_the_texts_size(bn, td, lengths, new, spare):
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(vocab=128)
    rng = np.random.default_rng(new)
    prompts = [rng.integers(0, 7, n).tolist() for n in lengths]
    n_pages = sum(_pages(p, new) for p in prompts) + spare
    dec = bn.StepDecoder(shape, bn.random_weights(shape, 9), n_pages=n_pages, max_seqs=len(prompts), max_ctx=300)
    weights = dec.w
    for max_nodes, draft in ((1, td.lookup_tree), (40, td.lookup_tree), (40, _wide), (64, _wide)):
        out, steps = td.tree_decode(dec, prompts, new, max_nodes=max_nodes, draft=draft, temperature=0.0)
        assert [len(t) for t in out] == [new] * len(prompts) and steps <= new
        assert dec.pool.table.free_pages == n_pages
        for p, t in zip(prompts, out):
            _greedy_or_near(bn, shape, weights, p, t, gs)


def test_rejected_drafts_give_their_pages_back(bn, td):
    """When a step's drafts are made, a sequence holds the pages of its cached tokens and no more."""
    shape = bn.Shape(vocab=128)
    dec = bn.StepDecoder(shape, bn.random_weights(shape, 9), n_pages=12, max_seqs=1, max_ctx=300)
    held = []

    def draft(history, max_nodes, depth, ngram):
        held.append((len(history), 12 - dec.pool.table.free_pages))
        return _wide(history, max_nodes, depth, ngram)
    td.tree_decode(dec, [[3] * 50], 20, max_nodes=64, temperature=0.0, draft=draft)
    assert len(held) > 2
    for length, pages in held:
        assert pages == -(-(length - 1) // 64)


def test_a_pool_too_small_for_the_texts_is_refused(bn, td):
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(vocab=128)
    dec = bn.StepDecoder(shape, bn.random_weights(shape, 9), n_pages=3, max_seqs=2, max_ctx=300)
    with pytest.raises(gs.GsError) as e:
        td.tree_decode(dec, [[1] * 60, [2] * 60], 60, max_nodes=16, temperature=0.0)
    assert e.value.code == gs.GS_ERR_OOM and dec.pool.table.free_pages == 3
