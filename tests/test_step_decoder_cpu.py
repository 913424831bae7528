"""Checks of best_of_n.py that need no GPU: what is refused before any device
work."""
import contextlib
import types

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def bn():
    from paper_2609_26638_gb300 import build
    build.build()
    from paper_2609_26638_gb300 import best_of_n
    return best_of_n


def _refused(bn, f, *args, **kw):
    with pytest.raises(bn.gs.GsError) as e:
        f(*args, **kw)
    assert e.value.code == bn.gs.GS_ERR_INVALID_ARG


def test_token_ids(bn):
    for good in ([0], [99, 0], np.array([5, 99]), torch.tensor([1, 2], dtype=torch.int32)):
        bn.check_tokens(good, 100)
    for bad in ([100], [-1], [3, 2 ** 40], np.array([0, 100]), torch.tensor([-5]), [1.0], [[1]],
                torch.tensor(3)):
        _refused(bn, bn.check_tokens, bad, 100)


def test_runs(bn):
    """Runs of one call name each place at most once."""
    for good, rows in (([(0, 0, [1, 2, 3])], 3), ([(0, 0, [1]), (1, 0, [1])], 2),
                       ([(0, 5, [1, 2]), (1, 3, [4]), (0, 7, [3, 4])], 5),
                       ([(0, 7, [3, 4]), (0, 5, [1, 2])], 4)):
        assert bn.check_runs(good, 5) == rows
    for bad in ([], [(0, 0, [])], [(0, 0, [1]), (1, 0, [])], [(0, 0, [1] * 6)],
                [(0, 0, [1, 2, 3]), (0, 2, [1])], [(0, 2, [1]), (1, 2, [1]), (0, 0, [1, 2, 3])],
                [(0, 4, [1]), (0, 4, [1])]):
        _refused(bn, bn.check_runs, bad, 5)


def test_uniforms(bn):
    """Any layout and type of the right shape becomes contiguous fp32 on the device."""
    g = torch.Generator().manual_seed(0)
    u = torch.rand(3, 5, generator=g)
    for given in (u, u.double(), u.t().contiguous().t(), torch.cat([u, u], 1)[:, :5], u.numpy(),
                  u.tolist()):
        got = bn.uniform_table(given, 3, 5, torch.device("cpu"))
        assert got.dtype == torch.float32 and got.is_contiguous() and torch.equal(got, u)
    assert bn.uniform_table(torch.empty(0, 5), 0, 5, torch.device("cpu")).shape == (0, 5)
    for bad in (u.t(), u[:2], u[:, :4], u[0], u[None], torch.tensor(0.5)):
        _refused(bn, bn.uniform_table, bad, 3, 5, torch.device("cpu"))


def test_sampler_checks_what_it_passes_on(bn, monkeypatch):
    """Logits and uniforms that do not fit the sampler's arrays, or that the
    kernel would read as something else, are refused; the type follows the logits."""
    gs = bn.gs
    calls = []
    monkeypatch.setattr(gs, "gs_sample", lambda *a: calls.append(a))

    @contextlib.contextmanager
    def within(stream):
        yield
    monkeypatch.setattr(torch.cuda, "stream", within)
    stream = types.SimpleNamespace(cuda_stream=3)
    s = bn.Sampler(4, top_k=7, device="cpu")
    x, u = torch.zeros(4, 100, dtype=torch.float16), torch.zeros(4)
    wide = torch.zeros(4, 128, dtype=torch.bfloat16)
    for logits, uni, code in ((x, u, gs.GS_F16), (wide[:, :100], u, gs.GS_BF16),
                              (x.float(), u, gs.GS_F32), (x[:2], u[:2], gs.GS_F16)):
        s.draw(logits, uni, stream)
        a = calls.pop()
        assert a[:5] == (logits.data_ptr(), logits.stride(0), len(logits), 100, code)
    one = x[:1].expand(4, -1)                            # every row the same memory: no row stride
    for logits, uni in ((x.double(), u), (x[0], u), (x.t().contiguous().t(), u), (one, u),
                        (torch.cat([x, x]), torch.zeros(8)), (x, u[:3]), (x, torch.zeros(5)),
                        (x, u.double()), (x, torch.zeros(8)[::2]), (x, u[:, None]),
                        (x.to("meta"), u), (x, u.to("meta"))):
        _refused(bn, s.draw, logits, uni, stream)
    assert not calls


def test_weights(bn):
    """Weights reach the kernels as pointers: type, shape, layout and device are checked."""
    shape = bn.Shape(n_layers=2, vocab=128)
    device = torch.device("cpu")

    def fresh():
        return bn.random_weights(shape, 0, "cpu")
    bn.check_weights(shape, fresh(), device)
    names = {"embed", "norm", "lm_head"} | {"layers"}
    assert set(fresh()) == names
    cases = [(None, k) for k in ("embed", "norm", "lm_head")] + \
        [(i, k) for i in (0, 1) for k in fresh()["layers"][0]]
    for layer, k in cases:
        t = (fresh() if layer is None else fresh()["layers"][layer])[k]
        wrong = [t.float(), t[:-1].contiguous(), t[None], t.to("meta"), None,
                 t.new_zeros(t.numel() + 1)[1:].view(t.shape)]          # 2 bytes off
        if t.dim() == 2:
            wrong += [t.new_zeros(t.shape[1], t.shape[0]).t(), t.new_zeros(t.shape[0], t.shape[1] + 8)[:, 8:]]
        for bad in wrong:
            w = fresh()
            (w if layer is None else w["layers"][layer])[k] = bad
            _refused(bn, bn.check_weights, shape, w, device)
    w = fresh()
    del w["layers"][1]
    _refused(bn, bn.check_weights, shape, w, device)
    w = fresh()
    del w["layers"][0]["o"]
    _refused(bn, bn.check_weights, shape, w, device)
