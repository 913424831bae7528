"""PagePool's device work without a device: on which stream each step runs.

torch.cuda.stream also makes the stream's device the current one, so what runs
within it works on a pool of any device; what runs outside goes to the current
device and stream of whoever calls."""
import contextlib
import types

import pytest
import torch


class _Err:
    """An error word that notes where it is read and cleared."""

    def __init__(self, log, word):
        self.log, self.word = log, word

    def item(self):
        self.log.append("item")
        return self.word

    def zero_(self):
        self.log.append("zero")
        self.word = 0

    def data_ptr(self):
        return 64


@pytest.fixture
def pool(monkeypatch):
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import cache, gs
    log = []
    stream = types.SimpleNamespace(cuda_stream=7, synchronize=lambda: log.append("synchronize"))

    @contextlib.contextmanager
    def within(s):
        assert s is stream
        log.append("enter")
        yield
        log.append("leave")
    p = cache.PagePool.__new__(cache.PagePool)
    p._torch = types.SimpleNamespace(cuda=types.SimpleNamespace(stream=within), tensor=torch.tensor,
                                     from_numpy=torch.from_numpy, int32=torch.int32)
    p.table = cache.PageTable(8, 4, 256)
    p.device, p.stream = torch.device("cpu"), stream
    p.kv = torch.zeros(1, 8, 2, 1, 64 * 64, dtype=torch.float16)
    p.rows = torch.zeros(p.table.rows.shape, dtype=torch.int32)
    p.err = _Err(log, 0)
    monkeypatch.setattr(gs, "gs_pages_copy", lambda *a: log.append("copy"))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    p.log = log
    return p


def _inside(log, what):
    """Every `what` of the log lies between an enter and its leave."""
    depth, at = 0, []
    for x in log:
        depth += (x == "enter") - (x == "leave")
        if x == what:
            at.append(depth)
    assert at
    return all(at)


def test_copies_run_within_the_pools_stream(pool):
    a = pool.open()
    pool.prepare([(a, 0, 100)])
    b, = pool.fork(a)
    pool.prepare([(b, 90, 1)])                       # copies the shared page
    assert _inside(pool.log, "copy")
    del pool.log[:]
    pool.close(a)
    pool.compact()
    assert _inside(pool.log, "copy")


def test_check_reads_and_clears_within_the_pools_stream(pool):
    """A word cleared on another stream could take a later kernel's report with it."""
    from paper_2609_26638_gb300 import gs
    pool.check()
    pool.err.word = 1
    with pytest.raises(gs.GsError) as e:
        pool.check()
    assert e.value.code == gs.GS_ERR_DEVICE_CHECK
    assert pool.log.count("synchronize") == 2 and pool.err.word == 0
    assert _inside(pool.log, "item") and _inside(pool.log, "zero")
    pool.check()
