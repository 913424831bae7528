"""best_of_n and its pool: what a failed call leaves behind, and each row's keys
against the whole forward in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_gpu_best_of_n import DEV, _decoder, _forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


def _prompt(n, seed=1):
    return np.random.default_rng(seed).integers(0, 4096, n).tolist()


def test_a_failed_call_gives_everything_back(bn, monkeypatch):
    """The pool too small, too few rows, too many tokens, a bad id, an error in
    a kernel: no page and no sequence stays taken, and the next call works."""
    from paper_2609_26638_gb300 import gs
    dec = _decoder(bn, bn.Shape(), n_pages=12, max_seqs=4, max_rows=70, max_ctx=400)
    want = bn.best_of_n(dec, _prompt(40), 3, 4, seed=2)[0].clone()

    def clean():
        assert dec.pool.table.free_pages == 12 and not dec.pool.table._pages
        assert torch.equal(bn.best_of_n(dec, _prompt(40), 3, 4, seed=2)[0], want)

    def fails(code, *args, **kw):
        with pytest.raises(gs.GsError) as e:
            bn.best_of_n(dec, *args, **kw)
        assert e.value.code == code
        clean()

    fails(gs.GS_ERR_INVALID_ARG, _prompt(390), 1, 40)            # past max_ctx
    fails(gs.GS_ERR_OOM, _prompt(380), 4, 10)                    # forks need more pages than there are
    fails(gs.GS_ERR_OOM, _prompt(10), 5, 2)                      # more rows than the table has
    fails(gs.GS_ERR_INVALID_ARG, _prompt(10), 71, 2)             # more than one feed takes
    fails(gs.GS_ERR_INVALID_ARG, _prompt(100) + [4096], 2, 2)    # in the prompt's second part
    real = dec.pool.prepare
    calls = []

    def prepare(spans):
        calls.append(1)
        if len(calls) == 3:
            with torch.cuda.stream(dec.stream):
                dec.pool.err.fill_(1)                            # as a kernel would
        return real(spans)
    monkeypatch.setattr(dec.pool, "prepare", prepare)
    fails(gs.GS_ERR_DEVICE_CHECK, _prompt(10), 2, 5)
    assert len(calls) > 4


def test_uniforms_of_any_layout(bn):
    """On the host, in 64 bits or transposed: the same draws."""
    from paper_2609_26638_gb300 import gs
    dec = _decoder(bn, bn.Shape())
    u = torch.rand(6, 3, generator=torch.Generator().manual_seed(4))
    want, total = (t.clone() for t in bn.best_of_n(dec, _prompt(33), 3, 6, uniforms=u.to(DEV)))
    for given in (u, u.double(), u.to(DEV).double(), u.to(DEV).t().contiguous().t(), u.numpy()):
        tokens, t2 = bn.best_of_n(dec, _prompt(33), 3, 6, uniforms=given)
        assert torch.equal(tokens, want) and torch.equal(t2, total)
    with pytest.raises(gs.GsError):
        bn.best_of_n(dec, _prompt(33), 3, 6, uniforms=u.t().contiguous())
    assert dec.pool.table.free_pages == 60


@pytest.mark.parametrize("plen", [130, 128, 63])
def test_every_row_of_a_shared_run(bn, plen):
    """Each of five continuations, step by step over shared pages that begin
    within a page, at its start and at its last slot: the logits after every
    token are those of the whole forward of that row's own tokens in 64 bits
    (3e-2, the tolerance of test_gpu_best_of_n.py), and best_of_n's tokens are the draws
    from them.  A page that a row shared and another wrote would show in the
    first, whichever row it is: one key of a neighbour's in place of its own moves
    a row's logits by 0.22 (prompt of 130, two tokens later)."""
    from paper_2609_26638_gb300 import gs
    shape, n, new = bn.Shape(), 5, 12
    prompt = _prompt(plen, seed=plen)
    u = torch.rand(new, n, generator=torch.Generator().manual_seed(2)).to(DEV)
    kw = dict(temperature=0.9, top_p=0.9, top_k=200)
    dec = _decoder(bn, shape)
    tokens, total = bn.best_of_n(dec, prompt, n, new, uniforms=u, **kw)
    host = tokens.cpu().numpy()
    assert len({tuple(r) for r in host[:, :4].tolist()}) == n    # rows part early: each its own keys
    want = [_forward(bn, shape, dec.w, np.concatenate([prompt, host[j]]), gs) for j in range(n)]
    sampler = bn.Sampler(n, **kw)
    stream = torch.cuda.current_stream()
    root = dec.pool.open()
    logits = dec.feed([(root, 0, prompt)])
    seqs = [root] + dec.pool.fork(root, n - 1)
    logits = logits.expand(n, -1).contiguous()
    mass = torch.zeros(n, device=DEV)
    for i in range(new):
        got = logits.cpu().double().numpy()
        for j in range(n):
            assert np.abs(got[j] - want[j][plen + i - 1]).max() <= 3e-2, (i, j)
        sampler.draw(logits, u[i], stream)
        assert torch.equal(sampler.token, tokens[:, i]), i
        mass += sampler.logprob
        logits = dec.feed([(q, plen + i, host[j, i: i + 1].tolist()) for j, q in enumerate(seqs)])
    got = logits.cpu().double().numpy()
    for j in range(n):
        assert np.abs(got[j] - want[j][plen + new - 1]).max() <= 3e-2, j
    assert torch.equal(mass, total)
    dec.check()
