"""PageTable.prepare with several spans of one sequence."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def cache():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import cache as module
    return module


def _state(t):
    return t.rows.copy(), t.refs.copy(), t.free_pages, {s: t.pages(s) for s in t._pages}


def _same(a, b):
    return np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1]) and a[2:] == b[2:]


@pytest.mark.parametrize("spans,pages", [
    ([(0, 64), (64, 10)], 2),
    ([(0, 100), (100, 100), (200, 1)], 4),
    ([(0, 1), (1, 1), (2, 200)], 4),
    ([(0, 130), (10, 5), (128, 70)], 4),
])
def test_a_span_may_start_where_the_one_before_ends(cache, spans, pages):
    t = cache.PageTable(10, 3, 300)
    s = t.open()
    assert t.prepare([(s, f, n) for f, n in spans]) == []
    assert len(t.pages(s)) == pages and t.free_pages == 10 - pages
    # the same slots again, as a holder among two: its pages are copied once each
    f, = t.fork(s)
    pairs = t.prepare([(f, a, n) for a, n in spans])
    assert sorted(p for p, _ in pairs) == sorted(t.pages(s))
    assert not set(t.pages(f)) & set(t.pages(s))


def test_gaps_are_still_refused_and_change_nothing(cache):
    from paper_2609_26638_gb300 import gs
    t = cache.PageTable(10, 3, 300)
    s, other = t.open(), t.open()
    t.prepare([(s, 0, 10)])
    before = _state(t)
    for spans in ([(s, 65, 1)], [(s, 10, 60), (s, 129, 1)], [(s, 128, 1), (s, 64, 64)],
                  [(s, 0, 64), (other, 64, 1)], [(s, 64, 64), (s, 128, 200)]):
        with pytest.raises(gs.GsError) as e:
            t.prepare(spans)
        assert e.value.code == gs.GS_ERR_INVALID_ARG
        assert _same(before, _state(t))
    # too few pages for the later span: nothing of the earlier ones either
    t.prepare([(other, 0, 300)])
    f, = t.fork(s)
    t.prepare([(f, 0, 200)])
    before = _state(t)
    with pytest.raises(gs.GsError) as e:
        t.prepare([(s, 64, 64), (s, 128, 64)])
    assert e.value.code == gs.GS_ERR_OOM and _same(before, _state(t))
