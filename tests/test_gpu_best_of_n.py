"""The sampled continuations of one prompt, end to end: logits of a fed token
against the whole forward in 64 bits, and continuations that do not depend on
whether their prompt's pages are shared."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


def _decoder(bn, shape, **kw):
    return bn.StepDecoder(shape, bn.random_weights(shape, 3), **{**dict(n_pages=60, max_seqs=8,
                                                                        max_ctx=400), **kw})


def _forward(bn, shape, w, tokens, gs):
    """Logits of every position, float64 on the host, straight from the formulas."""
    def f(t):
        return t.cpu().double().numpy()

    def norm(x, g):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + bn.EPS) * f(g)

    s, D = shape, shape.head_dim
    T = len(tokens)
    h = f(w["embed"])[tokens]
    half = s.rotary_dim // 2
    ang = np.arange(T)[:, None] * s.rope_theta ** (-2.0 * np.arange(half) / s.rotary_dim)
    i = np.arange(half)
    a, b = (i, i + half) if s.rope_layout == gs.ROPE_HALF else (2 * i, 2 * i + 1)

    def turn(x):
        y = x.copy()
        c, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * sn
        y[..., b] = x[..., b] * c + x[..., a] * sn
        return y

    for L in w["layers"]:
        x = (norm(h, L["norm1"]) @ f(L["qkv"]).T).reshape(T, -1, D)
        q = turn(norm(x[:, : s.n_heads], L["q_gain"]))
        k = turn(norm(x[:, s.n_heads: s.n_heads + s.n_kv_heads], L["k_gain"]))
        v = x[:, s.n_heads + s.n_kv_heads:]
        g = s.n_heads // s.n_kv_heads
        sc = np.einsum("thd,shd->hts", q, np.repeat(k, g, 1)) / np.sqrt(D)
        sc = np.where(np.tril(np.ones((T, T), bool)), sc, -np.inf)
        p = np.exp(sc - sc.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        h = h + np.einsum("hts,shd->thd", p, np.repeat(v, g, 1)).reshape(T, -1) @ f(L["o"]).T
        gu = norm(h, L["norm2"]) @ f(L["gate_up"]).T
        gate, up = gu[:, : s.d_ffn], gu[:, s.d_ffn:]
        h = h + (gate / (1 + np.exp(-gate)) * up) @ f(L["down"]).T
    return norm(h, w["norm"]) @ f(w["lm_head"]).T


@pytest.mark.parametrize("layout,D", [("INTERLEAVED", 64), ("HALF", 128)])
def test_logits_match_the_whole_forward(bn, layout, D):
    """A prompt in chunks and tokens one by one.  fp16 activations (2^-11 each)
    over two layers of O(1) activations and logits of size about 5: 3e-2, the
    tolerance of the engine's logits."""
    from paper_2609_26638_gb300 import gs
    shape = bn.Shape(head_dim=D, rope_layout=getattr(gs, "ROPE_" + layout), rotary_dim=D // 2)
    dec = _decoder(bn, shape, max_rows=70)
    tokens = np.random.default_rng(0).integers(0, shape.vocab, 150)
    want = _forward(bn, shape, dec.w, tokens, gs)
    seq = dec.pool.open()
    at = 0
    for chunk in (70, 1, 1, 57, 1, 20):
        got = dec.feed([(seq, at, tokens[at: at + chunk].tolist())])
        at += chunk
        dec.check()
        assert np.abs(got[0].cpu().double().numpy() - want[at - 1]).max() <= 3e-2, at


def test_continuations(bn):
    """n continuations over shared pages are those of n separate decodes with
    the same uniforms, up to draws at an edge of a token's interval: the first
    difference of a row must come with near-equal log-probabilities before it."""
    shape = bn.Shape()
    prompt = np.random.default_rng(1).integers(0, shape.vocab, 130).tolist()
    u = torch.rand(12, 5, generator=torch.Generator().manual_seed(2)).to(DEV)
    kw = dict(temperature=0.9, top_p=0.9, top_k=200)
    dec = _decoder(bn, shape)
    tokens, total = bn.best_of_n(dec, prompt, 5, 12, uniforms=u, **kw)
    assert dec.pool.table.free_pages == 60              # everything was given back
    again, total2 = bn.best_of_n(dec, prompt, 5, 12, uniforms=u, **kw)
    assert torch.equal(tokens, again) and torch.equal(total, total2)
    assert len({tuple(r) for r in tokens.tolist()}) > 1
    same = 0
    for j in range(5):
        one, t1 = bn.best_of_n(_decoder(bn, shape), prompt, 1, 12, uniforms=u[:, j: j + 1].contiguous(),
                               **kw)
        same += bool(torch.equal(one[0], tokens[j]))
        if torch.equal(one[0], tokens[j]):
            assert abs(float(t1[0]) - float(total[j])) < 12 * 3e-2
    assert same >= 4


def test_greedy_is_the_argmax(bn):
    shape = bn.Shape()
    dec = _decoder(bn, shape)
    prompt = list(range(40))
    tokens, total = bn.best_of_n(dec, prompt, 2, 6, temperature=0.0)
    assert torch.equal(tokens[0], tokens[1]) and (total == 0).all()
    seq = dec.pool.open()
    logits = dec.feed([(seq, 0, prompt)])
    for i in range(6):
        dec.check()
        assert int(tokens[0, i]) == int(logits[0].float().argmax())
        logits = dec.feed([(seq, 40 + i, [int(tokens[0, i])])])
    dec.check()
