"""StepDecoder as a caller uses it: streams, token ids, error words, refusals."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SLEEP = 40_000_000           # cycles: about 20 ms, a bounded spin


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


def _decoder(bn, shape=None, weights=None, **kw):
    shape = shape or bn.Shape()
    weights = weights or bn.random_weights(shape, 3)
    return bn.StepDecoder(shape, weights, **{**dict(n_pages=60, max_seqs=8, max_ctx=400), **kw})


def _prompt(n, vocab=4096, seed=5):
    return np.random.default_rng(seed).integers(0, vocab, n).tolist()


@pytest.mark.parametrize("side", [False, True])
def test_logits_are_ordered_behind_the_callers_stream(bn, side):
    """The last product comes late; the caller's stream reads the logits without
    synchronising, frees them, and reads the next call's."""
    dec = _decoder(bn)
    a, b = _prompt(30), _prompt(30, seed=6)
    want = []
    for p in (a, b):
        seq = dec.pool.open()
        want.append(dec.feed([(seq, 0, p)]).clone())
        dec.check()
    linear = dec._linear

    def late(x, w, *args):
        if w is dec.w["lm_head"]:
            torch.cuda._sleep(SLEEP)
        linear(x, w, *args)
    dec._linear = late
    stream = torch.cuda.Stream() if side else torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        got = []
        for p in (a, b):
            seq = dec.pool.open()
            logits = dec.feed([(seq, 0, p)])
            got.append(logits.clone())
            del logits
    stream.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    dec.check()


def test_tokens_are_read_behind_the_callers_stream(bn):
    """A token that the caller's stream has yet to write, freed right after the call."""
    dec = _decoder(bn)
    prompt = _prompt(20)
    one, two = dec.pool.open(), dec.pool.open()
    dec.feed([(one, 0, prompt), (two, 0, prompt)])
    want = dec.feed([(one, 20, [77])]).clone()
    dec.check()
    token = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    token += 77
    logits = dec.feed([(two, 20, token)])
    del token
    torch.full((1,), 5, dtype=torch.int32, device=DEV)         # may take the freed place
    dec.check()
    assert torch.equal(logits, want)


def test_best_of_n_on_a_side_stream(bn):
    """Uniforms that the caller's stream has yet to write; results used there."""
    dec = _decoder(bn)
    prompt = _prompt(70)
    u = torch.rand(5, 3, generator=torch.Generator().manual_seed(1)).to(DEV)
    want, total = bn.best_of_n(dec, prompt, 3, 5, uniforms=u)
    want, total = want.clone(), total.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        late = torch.zeros_like(u)
        torch.cuda._sleep(SLEEP)
        late += u
        got, t2 = bn.best_of_n(dec, prompt, 3, 5, uniforms=late)
        assert torch.equal(got, want) and torch.equal(t2, total)


def test_token_ids_outside_the_vocabulary(bn):
    """On the host: refused, and nothing has changed.  On the device: clamped,
    and the next check raises, once."""
    from paper_2609_26638_gb300 import gs
    dec = _decoder(bn)
    V = dec.shape.vocab
    seq = dec.pool.open()
    free = dec.pool.table.free_pages
    for bad in ([V], [-1], [3, 2 ** 40], np.array([V, 0])):
        with pytest.raises(gs.GsError) as e:
            dec.feed([(seq, 0, bad)])
        assert e.value.code == gs.GS_ERR_INVALID_ARG
        assert dec.pool.table.free_pages == free
    dec.check()
    for bad, inside in ((V, V - 1), (-1, 0), (-2 ** 31, 0), (2 ** 31 - 1, V - 1)):
        got = dec.feed([(seq, 0, torch.tensor([5, bad], dtype=torch.int32, device=DEV))]).clone()
        with pytest.raises(gs.GsError) as e:
            dec.check()
        assert e.value.code == gs.GS_ERR_DEVICE_CHECK
        dec.check()
        assert torch.equal(got, dec.feed([(seq, 0, [5, inside])]))
        dec.check()


def test_a_row_without_logits_is_reported(bn):
    """A language-model head of NaN: every draw is -1, which is no token to go on with."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape()
    w = bn.random_weights(shape, 3)
    w["lm_head"].fill_(float("nan"))
    dec = _decoder(bn, shape, w)
    with pytest.raises(gs.GsError) as e:
        bn.best_of_n(dec, _prompt(9), 2, 4)
    assert e.value.code == gs.GS_ERR_DEVICE_CHECK


@pytest.mark.parametrize("which", ["qkv", "gate_up", "lm_head"])
def test_a_product_beyond_fp16_is_reported(bn, which):
    """Any product of a step, not the last one alone, and feeds after it do not hide it."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape()
    w = bn.random_weights(shape, 3)
    m = w["lm_head"] if which == "lm_head" else w["layers"][0][which]
    good = m.clone()
    m.copy_(m.float().sign().half() * 60000)
    dec = _decoder(bn, shape, w)
    seq = dec.pool.open()
    dec.feed([(seq, 0, _prompt(9))])
    dec.stream.synchronize()
    m.copy_(good)
    torch.cuda.synchronize()
    dec.feed([(seq, 9, [3])])
    with pytest.raises(gs.GsError) as e:
        dec.check()
    assert e.value.code == gs.GS_ERR_DEVICE_CHECK
    dec.check()                                    # reported once
    dec.feed([(seq, 0, _prompt(9))])
    dec.check()


def test_one_check_clears_every_word(bn):
    from paper_2609_26638_gb300 import gs
    dec = _decoder(bn)
    for words in ("pa", "ag", "pg", "pag"):
        with torch.cuda.stream(dec.stream):
            for x in words:
                {"p": dec.pool.err, "a": dec.attn_scratch[:4].view(torch.int32), "g": dec.gemm_err}[x].fill_(1)
        with pytest.raises(gs.GsError):
            dec.check()
        dec.check()


def test_a_prompt_in_two_runs(bn):
    dec = _decoder(bn)
    p = _prompt(90)
    one, two = dec.pool.open(), dec.pool.open()
    want = dec.feed([(one, 0, p)])
    got = dec.feed([(two, 0, p[:33]), (two, 33, p[33:])])
    dec.check()
    assert torch.equal(got[1], want[0])
