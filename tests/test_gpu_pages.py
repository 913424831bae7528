"""gs_pages_copy and PagePool: copies are exact, whatever the sizes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gs():
    from paper_2609_26638_gb300 import gs as binding
    return binding


def _copy(gs, src, dst, pairs, stream=None):
    ids = torch.tensor(pairs, dtype=torch.int32, device=DEV).view(-1, 2).t().contiguous()
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    gs.gs_pages_copy(src.data_ptr(), src.shape[1], dst.data_ptr(), dst.shape[1], src.shape[0],
                     src.shape[2], ids[0].data_ptr() if len(pairs) else err.data_ptr(),
                     ids[1].data_ptr() if len(pairs) else err.data_ptr(), len(pairs), err.data_ptr(),
                     (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()
    return int(err.item())


@pytest.mark.parametrize("page_bytes", [16, 48, 4096, 16384, 16400, 262144])
@pytest.mark.parametrize("layers", [1, 3])
def test_copies(gs, page_bytes, layers):
    g = torch.Generator(device=DEV).manual_seed(page_bytes)
    pool = torch.randint(0, 256, (layers, 40, page_bytes), dtype=torch.uint8, device=DEV, generator=g)
    perm = np.random.default_rng(1).permutation(40)
    for pairs in ([], [(int(perm[0]), int(perm[1]))],
                  [(int(perm[0]), int(p)) for p in perm[1:8]],
                  list(zip(perm[:19].tolist(), perm[19:38].tolist()))):
        want = pool.clone()
        for s, d in pairs:
            want[:, d] = pool[:, s]
        assert _copy(gs, pool, pool, pairs, torch.cuda.Stream()) == 0
        assert torch.equal(pool, want)


def test_between_pools_and_bad_pages(gs):
    g = torch.Generator(device=DEV).manual_seed(0)
    src = torch.randint(0, 256, (2, 9, 1024), dtype=torch.uint8, device=DEV, generator=g)
    dst = torch.zeros(2, 5, 1024, dtype=torch.uint8, device=DEV)
    assert _copy(gs, src, dst, [(8, 0), (3, 4)]) == 0
    assert torch.equal(dst[:, 0], src[:, 8]) and torch.equal(dst[:, 4], src[:, 3])
    assert (dst[:, 1:4] == 0).all()
    for pair in ((9, 1), (-1, 1), (0, 5), (0, -1)):
        assert _copy(gs, src, dst, [pair, (1, 2)]) == 1
        assert torch.equal(dst[:, 2], src[:, 1]) and (dst[:, 1] == 0).all()


def test_more_pages_than_one_grid_holds(gs):
    n = 70000
    pool = torch.zeros(1, 2 * n, 16, dtype=torch.uint8, device=DEV)
    pool[0, :n] = (torch.arange(n, device=DEV)[:, None] % 251).to(torch.uint8)
    assert _copy(gs, pool, pool, np.stack([np.arange(n), n + np.arange(n)], 1).tolist()) == 0
    assert torch.equal(pool[0, :n], pool[0, n:])


def test_pool_forks_are_independent():
    """Each sequence's contents, written slot by slot through its own table row,
    survive forks, further writes, frees and compaction."""
    from paper_2609_26638_gb300.cache import PagePool
    side = torch.cuda.Stream()
    pool = PagePool(n_layers=2, n_pages=24, n_kv_heads=1, head_dim=64, dtype=torch.float16,
                    max_seqs=6, max_ctx=512, stream=side)
    rng = np.random.default_rng(2)
    want = {}

    def write(seq, first, count):
        pool.prepare([(seq, first, count)])
        with torch.cuda.stream(side):
            for t in range(first, first + count):
                v = float(rng.integers(1, 2000))
                page = int(pool.table.rows[seq, t // 64])
                pool.kv.view(2, 24, 2, 64, 64)[:, page, 0, t % 64] = v
                want[seq][t] = v

    def check():
        side.synchronize()
        rows = pool.rows.cpu().numpy()
        for seq, vals in want.items():
            for t, v in vals.items():
                got = pool.kv.view(2, 24, 2, 64, 64)[:, int(rows[seq, t // 64]), 0, t % 64]
                assert (got == v).all(), (seq, t)

    a = pool.open()
    want[a] = {}
    write(a, 0, 150)
    b, c = pool.fork(a, 2)
    want[b], want[c] = dict(want[a]), dict(want[a])
    check()
    write(b, 150, 70)
    write(a, 149, 2)
    write(c, 100, 1)
    check()
    pool.close(a)
    del want[a]
    assert pool.compact() == 24 - pool.table.free_pages
    check()
    d, = pool.fork(b)
    want[d] = dict(want[b])
    write(d, 10, 5)
    check()
    pool.check()
