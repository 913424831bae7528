"""Checks of the single-token step's operators that need no GPU: arguments are
refused before anything is launched, and the page bookkeeping holds its rules."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import gs as binding
    return binding


P = 1 << 12          # stands for a 16-byte aligned device address: never read on the host


def _cache(gs, **kw):
    v = dict(kv=P, n_pages=10, n_kv_heads=2, head_dim=64, dtype=gs.GS_F16, page_table=P, n_seq=3,
             pt_stride=8)
    v.update(kw)
    return gs.gs_cache(**v)


def _refused(gs, code, f, *args):
    with pytest.raises(gs.GsError) as e:
        f(*args)
    assert e.value.code == code


BAD_CACHES = [dict(kv=0), dict(kv=P + 8), dict(n_pages=0), dict(n_kv_heads=0), dict(page_table=0),
              dict(n_seq=0), dict(pt_stride=0), dict(dtype=2), dict(dtype=-1), dict(page_table=P + 2)]


def test_rope_append_refuses(gs):
    rope = gs.gs_rope(P, 100, 64, gs.ROPE_HALF)
    base = dict(qkv=P, ld=8 * 64, T=4, Hq=4, qg=P, kg=P, eps=1e-6, seq=P, slot=P, pos=P, q=2 * P,
                ldq=4 * 64, err=P, stream=0)

    def call(cache=None, rp=None, **kw):
        a = {**base, **kw}
        gs.gs_rope_append(cache or _cache(gs), rp or rope, *a.values())

    for bad in BAD_CACHES:
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(cache=_cache(gs, **bad)))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(cache=_cache(gs, head_dim=96)))
    for bad in ((0, 100, 64, 0), (P + 4, 100, 64, 0), (P, 0, 64, 0), (P, 100, 64, 2), (P, 100, 8, 0),
                (P, 100, 40, 0), (P, 100, 80, 0)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(rp=gs.gs_rope(*bad)))
    for bad in (dict(seq=P + 2), dict(slot=P + 1), dict(pos=P + 2), dict(err=P + 2), dict(qkv=0), dict(qkv=P + 2), dict(ld=8 * 64 - 8), dict(ld=8 * 64 + 4), dict(T=-1),
                dict(Hq=3), dict(Hq=0), dict(qg=0), dict(kg=0), dict(qg=P + 2), dict(eps=-1.0),
                dict(eps=float("nan")), dict(seq=0), dict(slot=0), dict(pos=0), dict(q=0),
                dict(ldq=4 * 64 - 8), dict(ldq=4 * 64 + 2), dict(err=0),
                dict(q=P)):          # over the projection, at another row stride
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    call(T=0)        # nothing to do


def test_rope_table_refuses(gs):
    def call(rot=64, rows=10, table=P, **kw):
        gs.gs_rope_table(gs.gs_rope_scaling(**{"kind": 0, "theta": 1e4, **kw}), rot, rows, table, 0)

    yarn = dict(kind=gs.ROPE_YARN, factor=2.0, original_ctx=10, beta_fast=32.0, beta_slow=1.0)
    for bad in (dict(rot=8), dict(rot=24), dict(rot=144), dict(rows=0), dict(table=0), dict(table=P + 4),
                dict(theta=0.0), dict(theta=float("inf")), dict(kind=4), dict(kind=-1),
                dict(kind=gs.ROPE_LINEAR, factor=0.5), dict(kind=gs.ROPE_NTK, factor=float("nan")),
                {**yarn, "original_ctx": 0}, {**yarn, "beta_fast": 0.5}, {**yarn, "beta_slow": 0.0},
                {**yarn, "magnitude": -1.0}):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))


def test_decode_attention_refuses(gs):
    base = dict(q=P, ldq=4 * 64, seq=0, n=P, rows=3, Hq=4, scale=0.125, window=0, out=P, ldo=4 * 64,
                lse=0, split=0, scratch=P, nb=1 << 30, stream=0)

    def call(cache=None, **kw):
        gs.gs_decode_attention(cache or _cache(gs), *{**base, **kw}.values())

    for bad in BAD_CACHES:
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(cache=_cache(gs, **bad)))
        assert gs.gs_decode_attention_scratch_bytes(_cache(gs, **bad), 3, 4, 0) == 0
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(cache=_cache(gs, head_dim=32)))
    for bad in (dict(q=0), dict(q=P + 2), dict(ldq=4 * 64 - 8), dict(ldq=4 * 64 + 4), dict(n=0),
                dict(rows=-1), dict(Hq=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(window=-1), dict(out=0), dict(out=P + 8),
                dict(ldo=4 * 64 - 8), dict(split=-1), dict(scratch=0), dict(scratch=P + 16),
                dict(seq=P + 2), dict(n=P + 2), dict(lse=P + 1)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(rows=65536, nb=1 << 60))
    need = gs.gs_decode_attention_scratch_bytes(_cache(gs), 3, 4, 0)
    assert need > 0
    _refused(gs, gs.GS_ERR_OOM, lambda: call(nb=need - 1))
    assert gs.gs_decode_attention_scratch_bytes(_cache(gs), 3, 4, 1) > \
        gs.gs_decode_attention_scratch_bytes(_cache(gs), 3, 4, 8)
    # the largest numbers are not added up
    most = 2 ** 31 - 1
    assert gs.gs_decode_attention_scratch_bytes(_cache(gs), 3, 4, most) == \
        gs.gs_decode_attention_scratch_bytes(_cache(gs), 3, 4, 8)
    call(rows=0, window=most, split=most)
    call(rows=0)


def test_sample_refuses(gs):
    p = gs.gs_sample_params(0, 0, 0, 0)
    base = dict(x=P, ld=1000, rows=2, vocab=1000, dt=gs.GS_BF16, params=p, u=P, token=P, logprob=0,
                kept=0, stream=0)

    def call(**kw):
        gs.gs_sample(*{**base, **kw}.values())

    for bad in (dict(x=0), dict(ld=999), dict(rows=-1), dict(vocab=0), dict(dt=3), dict(dt=-1),
                dict(u=0), dict(token=0), dict(x=P + 1), dict(x=P + 2, dt=gs.GS_F32), dict(u=P + 2),
                dict(token=P + 2), dict(logprob=P + 2), dict(kept=P + 1),
                dict(params=gs.gs_sample_params(P + 2, 0, 0, 0)),
                dict(params=gs.gs_sample_params(0, 0, 0, P + 1))):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(vocab=262145, ld=262145))
    call(rows=0)


def test_pages_copy_refuses(gs):
    base = dict(src=P, sp=4, dst=P, dp=4, layers=2, nb=4096, s=P, d=P, n=1, err=P, stream=0)

    def call(**kw):
        gs.gs_pages_copy(*{**base, **kw}.values())

    for bad in (dict(src=0), dict(src=P + 8), dict(dst=0), dict(dst=P + 4), dict(sp=0), dict(dp=0),
                dict(layers=0), dict(nb=0), dict(nb=24), dict(s=0), dict(d=0), dict(n=-1), dict(err=0),
                dict(s=P + 2), dict(d=P + 1), dict(err=P + 2)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(layers=65536))
    call(n=0)


# ------------------------------------------------------------------ pages
def test_page_table_rules(gs):
    """Random opens, forks, writes, truncations, closes and compactions against
    a model that keeps every sequence's contents: no write reaches another
    sequence, counts add up, and a refused call changes nothing."""
    from paper_2609_26638_gb300.cache import PAGE_TOKENS, PageTable
    rng = np.random.default_rng(0)
    t = PageTable(n_pages=40, max_seqs=7, max_ctx=700)
    store = np.full((40, PAGE_TOKENS), -1, dtype=np.int64)     # the pages' contents
    want = {}                                                  # sequence -> contents
    stamp = 0

    def check():
        held = np.zeros(40, dtype=np.int64)
        for s, vals in want.items():
            pages = t.pages(s)
            for p in pages:
                held[p] += 1
            assert list(t.rows[s, : len(pages)]) == pages
            got = store[pages].reshape(-1)[: len(vals)]
            assert np.array_equal(got, vals), s
        assert np.array_equal(held, t.refs)
        assert t.free_pages == int((held == 0).sum())

    def apply(pairs):
        assert not {a for a, _ in pairs} & {b for _, b in pairs}
        assert len({b for _, b in pairs}) == len(pairs)
        for a, b in pairs:
            store[b] = store[a]

    refused = 0
    for _ in range(3000):
        op = rng.choice(["open", "fork", "write", "write", "write", "truncate", "close", "compact"])
        live = list(want)
        s = int(rng.choice(live)) if live else None
        before = (t.rows.copy(), t.refs.copy(), t.free_pages)
        try:
            if op == "open":
                want[t.open()] = np.zeros(0, np.int64)
            elif s is None:
                continue
            elif op == "fork":
                for n in t.fork(s, int(rng.integers(0, 4))):
                    want[n] = want[s].copy()
            elif op == "write":
                spans = []
                for q in rng.choice(live, size=rng.integers(1, len(live) + 1), replace=False):
                    first = int(rng.integers(0, len(want[int(q)]) + 1))
                    spans.append((int(q), first, int(rng.integers(1, 90))))
                apply(t.prepare(spans))
                for q, first, count in spans:
                    vals = np.concatenate([want[q], np.full(max(0, first + count - len(want[q])), -1)])
                    stamp += 1
                    vals[first: first + count] = stamp * 1000 + np.arange(count)
                    want[q] = vals
                    pages = t.pages(q)
                    for i in range(first, first + count):
                        store[pages[i // 64], i % 64] = vals[i]
            elif op == "truncate":
                n = int(rng.integers(0, len(want[s]) + 1))
                t.truncate(s, n)
                want[s] = want[s][:n]
            elif op == "close":
                t.close(s)
                del want[s]
            else:
                apply(t.compact())
                used = int((t.refs > 0).sum())
                assert (t.refs[:used] > 0).all()
        except gs.GsError as e:
            refused += 1
            assert e.code in (gs.GS_ERR_OOM, gs.GS_ERR_INVALID_ARG)
            assert np.array_equal(before[0], t.rows) and np.array_equal(before[1], t.refs)
            assert before[2] == t.free_pages
        check()
    assert refused > 20


def test_page_table_refusals(gs):
    from paper_2609_26638_gb300.cache import PageTable
    t = PageTable(n_pages=4, max_seqs=2, max_ctx=200)
    with pytest.raises(ValueError):
        t.pages(0)
    s = t.open()
    for first, count in ((0, 0), (-1, 5), (0, 201), (65, 1)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, t.prepare, [(s, first, count)])
    t.prepare([(s, 0, 200)])
    _refused(gs, gs.GS_ERR_INVALID_ARG, t.truncate, s, 300)
    _refused(gs, gs.GS_ERR_OOM, t.fork, s, 2)
    f, = t.fork(s)
    _refused(gs, gs.GS_ERR_OOM, t.prepare, [(f, 100, 1)])
    _refused(gs, gs.GS_ERR_OOM, t.open)
    t.close(f)
    with pytest.raises(ValueError):
        t.close(f)
    with pytest.raises(ValueError):
        PageTable(0, 1, 1)
