"""Refusals of the operators for drafted trees and 4-bit weights: arguments are
checked before anything is launched, so these need no GPU."""
import pytest


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import gs as binding
    return binding


P = 1 << 12          # stands for an aligned device address: never read on the host


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


def test_tree_attention_refuses(gs):
    base = dict(q=P, ldq=4 * 64, seq=0, n=P, count=0, mask=P, pos=0, trees=3, nodes=5, Hq=4, scale=0.125,
                window=0, out=P, ldo=4 * 64, lse=0, split=0, scratch=P, nb=1 << 40, stream=0)

    def call(cache=None, **kw):
        gs.gs_tree_attention(cache or _cache(gs), *{**base, **kw}.values())

    for bad in BAD_CACHES:
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(cache=_cache(gs, **bad)))
        assert gs.gs_tree_attention_scratch_bytes(_cache(gs, **bad), 3, 5, 4, 0) == 0
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(cache=_cache(gs, head_dim=32)))
    for bad in (dict(q=0), dict(q=P + 2), dict(ldq=4 * 64 - 8), dict(ldq=4 * 64 + 4), dict(n=0),
                dict(mask=0), dict(mask=P + 4), dict(trees=-1), dict(nodes=0), dict(nodes=-3), dict(Hq=3),
                dict(Hq=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(window=-1), dict(window=5), dict(out=0), dict(out=P + 8),
                dict(ldo=4 * 64 - 8), dict(split=-1), dict(scratch=0), dict(scratch=P + 16),
                dict(seq=P + 2), dict(n=P + 2), dict(count=P + 1), dict(pos=P + 2), dict(lse=P + 1)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    for bad in (dict(nodes=65), dict(trees=65536), dict(Hq=1 << 14, ldq=1 << 20, ldo=1 << 20)):
        _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(**bad))
    for split in (0, 1, 3):
        need = gs.gs_tree_attention_scratch_bytes(_cache(gs), 3, 5, 4, split)
        assert need > 0
        _refused(gs, gs.GS_ERR_OOM, lambda: call(nb=need - 1, split=split))
    most = 2 ** 31 - 1
    assert gs.gs_tree_attention_scratch_bytes(_cache(gs), 3, 5, 4, most) == \
        gs.gs_tree_attention_scratch_bytes(_cache(gs), 3, 5, 4, 8)
    call(trees=0, window=most, pos=P, split=most)
    call(trees=0)


def test_tree_accept_refuses(gs):
    base = dict(parent=P, token=P, choice=P, count=0, most=0, eos=-1, trees=2, nodes=9, path=P, next=P,
                length=P, err=P, stream=0)

    def call(**kw):
        gs.gs_tree_accept(*{**base, **kw}.values())

    for bad in (dict(parent=0), dict(token=0), dict(choice=0), dict(path=0), dict(next=0), dict(length=0),
                dict(err=0), dict(trees=-1), dict(nodes=0), dict(parent=P + 2), dict(token=P + 1),
                dict(choice=P + 2), dict(count=P + 2), dict(most=P + 2), dict(path=P + 2),
                dict(next=P + 2), dict(length=P + 2), dict(err=P + 2)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(nodes=65))
    call(trees=0)


def test_tree_commit_refuses(gs):
    base = dict(layers=2, seq=0, n=P, path=P, length=P, trees=2, nodes=9, err=P, stream=0)

    def call(cache=None, **kw):
        gs.gs_tree_commit(cache or _cache(gs), *{**base, **kw}.values())

    for bad in BAD_CACHES:
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(cache=_cache(gs, **bad)))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(cache=_cache(gs, head_dim=96)))
    for bad in (dict(layers=0), dict(n=0), dict(path=0), dict(length=0), dict(err=0), dict(trees=-1),
                dict(nodes=0), dict(seq=P + 2), dict(n=P + 2), dict(path=P + 2), dict(length=P + 2),
                dict(err=P + 2)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    for bad in (dict(nodes=65), dict(layers=65536), dict(trees=65536)):
        _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(**bad))
    call(trees=0)


def _weight(gs, **kw):
    v = dict(packed=P, N=64, K=128, group=64, dtype=gs.GS_F16, zeros=0, gated=0)
    v.update(kw)
    return gs.gs_qweight(*v.values())


BAD_WEIGHTS = [dict(N=0), dict(N=-5), dict(K=0), dict(K=16), dict(K=96), dict(dtype=2), dict(dtype=-1),
               dict(zeros=2), dict(zeros=-1), dict(gated=2), dict(N=63, gated=1)]
UNSUPPORTED_WEIGHTS = [dict(group=16), dict(group=0), dict(group=256), dict(K=(1 << 20) + 64),
                       dict(N=(1 << 24) + 1)]


def test_qweight_refuses(gs):
    def pack(q=P, scale=P, zero=0, **kw):
        gs.gs_qweight_pack(_weight(gs, **kw), q, scale, zero, 0)

    for bad in BAD_WEIGHTS:
        assert gs.gs_qweight_bytes(_weight(gs, **bad)) == 0
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: pack(**bad))
    for bad in UNSUPPORTED_WEIGHTS:
        assert gs.gs_qweight_bytes(_weight(gs, **bad)) == 0
        _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: pack(**bad))
    for bad in (dict(packed=0), dict(packed=P + 8), dict(q=0), dict(q=P + 1), dict(scale=0),
                dict(scale=P + 1), dict(zero=P), dict(zeros=1)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: pack(**bad))
    # 16 rows of 128: weights, two bytes of scale and one of zero per group of 32
    assert gs.gs_qweight_bytes(_weight(gs, N=16, group=32)) == 16 * 64 + 16 * 4 * 2
    assert gs.gs_qweight_bytes(_weight(gs, N=16, group=32, zeros=1)) == 16 * 64 + 16 * 4 * 3


def test_qlinear_refuses(gs):
    base = dict(x=P, ldx=128, y=P, ldy=64, M=4, epi=gs.EPI_STORE_F16, err=P, stream=0)

    def call(weight={}, **kw):
        gs.gs_qlinear(_weight(gs, **weight), *{**base, **kw}.values())

    for bad in BAD_WEIGHTS + [dict(packed=0), dict(packed=P + 4), dict(gated=1)]:
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(weight=bad))
    for bad in UNSUPPORTED_WEIGHTS:
        _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(weight=bad))
    for bad in (dict(x=0), dict(x=P + 8), dict(ldx=120), dict(ldx=132), dict(y=0), dict(y=P + 1),
                dict(ldy=63), dict(M=-1), dict(epi=-1), dict(epi=3), dict(epi=gs.EPI_SWIGLU),
                dict(epi=gs.EPI_RESID_F32, y=P + 2), dict(err=0), dict(err=P + 2)):
        _refused(gs, gs.GS_ERR_INVALID_ARG, lambda: call(**bad))
    _refused(gs, gs.GS_ERR_UNSUPPORTED, lambda: call(M=(1 << 21) + 1))
    call(M=0)
    call(M=0, weight=dict(gated=1), epi=gs.EPI_SWIGLU, ldy=32)
