"""Drafted trees through a decoder, end to end: logits of every node and of what
follows the kept path against the whole forward in 64 bits, 4-bit weights, and the
decoding loop.

fp16 activations (2^-11 each) over two layers of O(1) activations and logits of size
about 5: 3e-2, the tolerance of the engine's logits."""
import numpy as np
import pytest
import torch

from tests.test_gpu_best_of_n import _forward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 3e-2


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


@pytest.fixture(scope="module")
def td():
    from paper_2609_26638_gb300 import tree_decode
    return tree_decode


def _plain(w):
    """The values of a decoder's weights, 4-bit ones as they were before packing."""
    def of(x):
        return x if isinstance(x, torch.Tensor) else x.plain
    return {**w, "layers": [{k: of(v) for k, v in layer.items()} for layer in w["layers"]],
            "lm_head": of(w["lm_head"])}


def _quantized(bn, shape, group, zeros, seed=3):
    from paper_2609_26638_gb300 import qweight
    w = bn.random_weights(shape, seed)
    out = qweight.quantize_decoder(w, group, zeros)

    def back(x, held):
        q, s, z = qweight.quantize(x, group, zeros)
        whole = torch.stack([q & 15, q >> 4], -1).flatten(1).double()
        zz = 8 if z is None else z.double().repeat_interleave(group, 1)
        held.plain = (whole - zz) * s.double().repeat_interleave(group, 1)
    for old, new in zip(w["layers"], out["layers"]):
        for k in ("qkv", "o", "gate_up", "down"):
            back(old[k], new[k])
    back(w["lm_head"], out["lm_head"])
    return out


def _tree(rng, nodes, vocab):
    return rng.integers(0, vocab, nodes).tolist(), [-1] + [int(rng.integers(0, i)) for i in range(1, nodes)]


def _path(parents, i):
    path = [i]
    while path[-1]:
        path.append(parents[path[-1]])
    return path[::-1]


@pytest.mark.parametrize("layout,D,heads,bits", [("INTERLEAVED", 64, (8, 2), 16), ("HALF", 128, (2, 2), 16),
                                                 ("HALF", 64, (8, 1), 4), ("HALF", 128, (4, 2), 4)])
def test_trees_match_the_whole_forward(bn, layout, D, heads, bits):
    """Trees of several sizes over several sequences, their paths kept, trees again."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(head_dim=D, n_heads=heads[0], n_kv_heads=heads[1],
                     rope_layout=getattr(gs, "ROPE_" + layout), rotary_dim=D // 2)
    weights = bn.random_weights(shape, 3) if bits == 16 else _quantized(bn, shape, 64, D == 64)
    dec = bn.StepDecoder(shape, weights, n_pages=60, max_seqs=8, max_ctx=400, max_rows=128)
    w = _plain(weights)
    rng = np.random.default_rng(D)
    text = [rng.integers(0, shape.vocab, n).tolist() for n in (1, 63, 130)]
    seqs = [dec.pool.open() for _ in text]
    for seq, t in zip(seqs, text):
        if len(t) > 1:
            dec.feed([(seq, 0, t[:-1])]) if len(t) < 129 else [dec.feed([(seq, a, t[a: min(a + 128, 129)])])
                                                               for a in (0, 128)]
    for nodes in ((1, 1, 1), (5, 2, 9), (17, 30, 40), (3, 40, 8)):
        trees = []
        for seq, t, m in zip(seqs, text, nodes):
            tokens, parents = _tree(rng, m, shape.vocab)
            tokens[0] = t[-1]
            trees.append((seq, len(t) - 1, tokens, parents))
        logits = dec.feed_trees(trees)
        dec.check()
        want = []
        for (_, n, tokens, parents), t, got in zip(trees, text, logits):
            per = {}
            for i in range(len(tokens)):
                leaf = _path(parents, i)
                if i not in set(parents) or len(tokens) == 1:      # a leaf: its whole path at once
                    out = _forward(bn, shape, w, t[:-1] + [tokens[j] for j in leaf], gs)
                    for d, j in enumerate(leaf):
                        per[j] = out[n + d]
            err = max(np.abs(got[i].cpu().double().numpy() - per[i]).max() for i in per)
            assert len(per) == len(tokens) and err <= TOL, (nodes, err)
            want.append(per)
        # choices that follow a path of each tree to a random node, then leave it
        choice = torch.full(logits.shape[:2], shape.vocab - 1, dtype=torch.int32)
        ends = []
        for b, (_, _, tokens, parents) in enumerate(trees):
            end = int(rng.integers(0, len(tokens)))
            path = _path(parents, end)
            for i, j in zip(path, path[1:]):
                choice[b, i] = tokens[j]
            ends.append([tokens[j] for j in path[1:]])
        got = dec.keep(trees, choice.to(DEV))
        dec.check()
        for t, new, end in zip(text, got, ends):
            assert new[: len(end)] == end and len(new) >= len(end) + 1    # (equal siblings may lead on)
            t += new


def _greedy_or_near(bn, shape, w, prompt, out, gs):
    """Every token is the whole forward's largest logit, or within the tolerance of it."""
    want = _forward(bn, shape, w, prompt + out, gs)
    for i, t in enumerate(out):
        row = want[len(prompt) - 1 + i]
        assert row.max() - row[t] <= 2 * TOL, i


def test_greedy_text(bn, td):
    """Greedy decoding with looked-up trees, of several prompts at once, is greedy."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(vocab=128)
    weights = bn.random_weights(shape, 5)
    dec = bn.StepDecoder(shape, weights, n_pages=40, max_seqs=4, max_ctx=300)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, 8, n).tolist() for n in (1, 40, 129)]
    free = dec.pool.table.free_pages
    for max_nodes in (1, 16, 40):
        out, steps = td.tree_decode(dec, prompts, 24, max_nodes=max_nodes, temperature=0.0)
        assert [len(t) for t in out] == [24] * 3 and steps <= 24
        assert dec.pool.table.free_pages == free
        for p, t in zip(prompts, out):
            _greedy_or_near(bn, shape, weights, p, t, gs)


def test_right_drafts_are_kept(bn, td):
    """Drafted with its own continuation, a step keeps all of the tree's depth."""
    shape = bn.Shape()
    dec = bn.StepDecoder(shape, bn.random_weights(shape, 6), n_pages=40, max_seqs=4, max_ctx=300)
    prompt = np.random.default_rng(2).integers(0, shape.vocab, 70).tolist()
    (text,), steps = td.tree_decode(dec, [prompt], 20, max_nodes=1, temperature=0.0)
    assert steps == 20
    whole = prompt + text

    def draft(history, max_nodes, depth, ngram):
        more = whole[len(history): len(history) + depth]
        return [history[-1], 5] + more, [-1, 0] + [0 if i == 0 else i + 1 for i in range(len(more))]
    (again,), steps = td.tree_decode(dec, [prompt], 20, depth=4, draft=draft, temperature=0.0)
    assert again == text and steps == 4


def test_texts_that_fill_the_context(bn, td):
    """Trees at the end of a table, cut to the room there, beside wide ones."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(vocab=128)
    weights = bn.random_weights(shape, 8)
    dec = bn.StepDecoder(shape, weights, n_pages=12, max_seqs=2, max_ctx=128)
    rng = np.random.default_rng(6)
    prompts = [rng.integers(0, 3, n).tolist() for n in (108, 60)]
    out, _ = td.tree_decode(dec, prompts, 20, max_nodes=40, ngram=1, temperature=0.0)
    assert [len(t) for t in out] == [20, 20]
    for p, t in zip(prompts, out):
        _greedy_or_near(bn, shape, weights, p, t, gs)


def test_sampled_text_does_not_depend_on_the_drafts(bn, td):
    """With the numbers of each position given, drafts change nothing; and an eos ends a text."""
    shape = bn.Shape()
    dec = bn.StepDecoder(shape, bn.random_weights(shape, 7), n_pages=40, max_seqs=4, max_ctx=300)
    rng = np.random.default_rng(3)
    prompts = [rng.integers(0, shape.vocab, n).tolist() for n in (30, 65)]
    u = torch.rand(2, 65 + 12, generator=torch.Generator().manual_seed(4))
    kw = dict(uniforms=u, temperature=0.7, top_k=3)
    want, steps = td.tree_decode(dec, prompts, 12, max_nodes=1, **kw)
    whole = [p + t for p, t in zip(prompts, want)]

    def draft(history, max_nodes, depth, ngram):
        full = next(w for w in whole if w[: len(history)] == history)
        more = full[len(history): len(history) + depth]
        return [history[-1]] + more, list(range(-1, len(more)))
    got, fewer = td.tree_decode(dec, prompts, 12, depth=3, draft=draft, **kw)
    assert got == want and steps == 12 and fewer == 3
    eos = want[0][5]
    got, _ = td.tree_decode(dec, prompts, 12, depth=3, draft=draft, eos=eos, **kw)
    for g, t in zip(got, want):
        end = t.index(eos) + 1 if eos in t else 12
        assert g == t[:end]


def test_quantized_decoder_feeds_tokens(bn):
    """A prompt and single tokens through 4-bit weights; range errors are reported."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape()
    weights = _quantized(bn, shape, 32, True)
    dec = bn.StepDecoder(shape, weights, n_pages=20, max_seqs=2, max_ctx=200)
    tokens = np.random.default_rng(5).integers(0, shape.vocab, 90)
    want = _forward(bn, shape, _plain(weights), tokens, gs)
    seq, at = dec.pool.open(), 0
    for chunk in (70, 1, 1, 17, 1):
        got = dec.feed([(seq, at, tokens[at: at + chunk].tolist())])
        at += chunk
        dec.check()
        assert np.abs(got[0].cpu().double().numpy() - want[at - 1]).max() <= TOL
    dec.w["norm"] *= 30000
    dec.feed([(seq, at, [5])])
    with pytest.raises(gs.GsError):
        dec.check()
    dec.check()


def test_refusals(bn, td):
    from paper_2609_26638_gb300 import gs, qweight
    shape = bn.Shape()
    dec = bn.StepDecoder(shape, bn.random_weights(shape), n_pages=3, max_seqs=2, max_ctx=128, max_rows=40)
    seq = dec.pool.open()
    tree = [(seq, 0, [1, 2], [-1, 0])]
    for bad in ([(seq, 0, [1, 4096], [-1, 0])], [(seq, 0, [1] * 41, list(range(-1, 40)))]):
        with pytest.raises(gs.GsError):
            dec.feed_trees(bad)
    dec.feed_trees(tree)
    for choice in (torch.zeros(1, 2, dtype=torch.int64, device=DEV), torch.zeros(1, 3, dtype=torch.int32, device=DEV),
                   torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, 1, dtype=torch.int32, device=DEV).t()[:, ::1]):
        if choice.shape == (1, 2) and choice.dtype == torch.int32 and choice.is_cuda and choice.is_contiguous():
            continue
        with pytest.raises(gs.GsError):
            dec.keep(tree, choice)
    with pytest.raises(gs.GsError):
        dec.keep(tree, torch.zeros(1, 2, dtype=torch.int32, device=DEV), most=[1, 1])
    with pytest.raises(gs.GsError):                       # more pages than the pool has
        td.tree_decode(dec, [[1] * 60, [2] * 60], 60, max_nodes=16, temperature=0.0)
    assert dec.pool.table.free_pages == 2
    wrong = bn.random_weights(shape)
    w = wrong["layers"][0]
    w["gate_up"] = qweight.QWeight(*qweight.quantize(w["gate_up"], 64), group=64)      # not gated
    with pytest.raises(gs.GsError):
        bn.StepDecoder(shape, wrong, n_pages=3, max_seqs=2, max_ctx=128)
