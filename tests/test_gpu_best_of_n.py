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


def test_graph_replay(bn):
    """The four operators captured in one graph: replays give the eager results."""
    from paper_2609_26638_gb300 import gs
    from paper_2609_26638_gb300.cache import PagePool
    g = torch.Generator(device=DEV).manual_seed(0)
    st = torch.cuda.Stream()
    pool = PagePool(n_layers=1, n_pages=8, n_kv_heads=2, head_dim=64, dtype=torch.float16, max_seqs=2,
                    max_ctx=256, stream=st)
    seq = pool.open()
    pool.prepare([(seq, 0, 100)])
    table = torch.empty(256, 32, 2, device=DEV)
    qkv = torch.randn(1, 8 * 64, device=DEV, generator=g).half()
    logits = torch.randn(1, 999, device=DEV, generator=g).half()
    i32 = [torch.tensor([v], dtype=torch.int32, device=DEV) for v in (seq, 99, 100, 0, 7)]
    u = torch.full((1,), 0.37, device=DEV)
    q, out = torch.zeros(2, 1, 4 * 64, dtype=torch.float16, device=DEV)
    token = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = pool.layer(0)
    scratch = torch.zeros(gs.gs_decode_attention_scratch_bytes(cache, 1, 4, 1), dtype=torch.uint8,
                          device=DEV)
    rope, par = gs.gs_rope(table.data_ptr(), 256, 64, gs.ROPE_HALF), gs.gs_sample_params(0, 0, 0, 0)
    gs.gs_rope_table(gs.gs_rope_scaling(kind=gs.ROPE_PLAIN, theta=1e4), 64, 256, table.data_ptr(),
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()

    def step():
        s = torch.cuda.current_stream().cuda_stream
        gs.gs_rope_append(cache, rope, qkv.data_ptr(), 8 * 64, 1, 4, 0, 0, 1e-6, i32[0].data_ptr(),
                          i32[1].data_ptr(), i32[1].data_ptr(), q.data_ptr(), 4 * 64,
                          pool.err.data_ptr(), s)
        gs.gs_decode_attention(cache, q.data_ptr(), 4 * 64, i32[0].data_ptr(), i32[2].data_ptr(), 1, 4,
                               0.125, 0, out.data_ptr(), 4 * 64, 0, 1, scratch.data_ptr(),
                               scratch.numel(), s)
        gs.gs_sample(logits.data_ptr(), 999, 1, 999, gs.GS_F16, par, u.data_ptr(), token.data_ptr(), 0,
                     0, s)
        gs.gs_pages_copy(pool.kv.data_ptr(), 8, pool.kv.data_ptr(), 8, 1, pool.kv[0, 0].numel() * 2,
                         i32[3].data_ptr(), i32[4].data_ptr(), 1, pool.err.data_ptr(), s)

    with torch.cuda.stream(st):
        step()
        st.synchronize()
        want = [t.clone() for t in (q, out, token, pool.kv)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            step()
        for t in (q, out, token):
            t.zero_()
        pool.kv[0, 7].zero_()
        graph.replay()
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (q, out, token, pool.kv)))
    assert (out != 0).any() and (pool.kv[0, 7] == pool.kv[0, 0]).all()


def test_greedy_is_the_argmax(bn):
    shape = bn.Shape()
    dec = _decoder(bn, shape)
    prompt = list(range(40))
    from paper_2609_26638_gb300 import gs
    for bad in (([], 2, 6), (prompt, 0, 6), (prompt, 2, -1)):
        with pytest.raises(gs.GsError):
            bn.best_of_n(dec, *bad)
    tokens, total = bn.best_of_n(dec, prompt, 2, 6, temperature=0.0)
    assert torch.equal(tokens[0], tokens[1]) and (total == 0).all()
    seq = dec.pool.open()
    logits = dec.feed([(seq, 0, prompt)])
    for i in range(6):
        dec.check()
        assert int(tokens[0, i]) == int(logits[0].float().argmax())
        logits = dec.feed([(seq, 40 + i, [int(tokens[0, i])])])
    dec.check()
