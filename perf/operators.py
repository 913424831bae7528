"""Cases and plain forms of the sampled single-token decoding operators.

Four operators make one sampled decoding step over a paged key-value cache:

  append  per-head RMS norm of queries and keys, rotary positions, and the
          write of keys and values into their cache pages (one pass)
  attend  attention of one new token per sequence over its pages
  sample  temperature, min-p, top-k and top-p, and the draw of a token from a
          given uniform number
  copy    copies of cache pages for forked sequences and for closing gaps

A page holds 64 tokens of one layer: [2][kv heads][64 * head_dim], keys as
[64 tokens][head_dim], values transposed as [head_dim][64 tokens].
"""
import numpy as np
import torch

own = False

PAGE = 64
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
MASS_ONE = float(2 ** 40)        # the integer weight of the most likely token
NEG_INF = float("-inf")


# ------------------------------------------------------------------- cases
def listed():
    return [
        # one sequence's next token in an unbatched decode: launch latency
        dict(name="append one token", op="append", dtype="fp16", tokens=1, seqs=1, first=200,
             heads=16, kv_heads=8, dim=64, rot=64, layout="half", norm=True),
        # a decode step of a large batch, each sequence at its own length
        dict(name="append batch 256", op="append", dtype="bf16", tokens=256, seqs=256, first=130,
             heads=16, kv_heads=8, dim=64, rot=32, layout="interleaved", norm=True),
        # packed prompts of odd lengths, the second chunk of each
        dict(name="append prompts 8191", op="append", dtype="bf16", tokens=8191, seqs=5, first=333,
             heads=32, kv_heads=8, dim=128, rot=128, layout="half", norm=True),
        # a short context, one sequence: latency
        dict(name="attend one short", op="attend", dtype="fp16", seqs=1, lo=517, hi=517,
             heads=16, kv_heads=8, dim=64, window=0),
        # the serving batch: 32 sequences of 1024 to 6144 tokens
        dict(name="attend serving 32", op="attend", dtype="fp16", seqs=32, lo=1024, hi=6144,
             heads=16, kv_heads=8, dim=64, window=0),
        # one very long document
        dict(name="attend one long", op="attend", dtype="bf16", seqs=1, lo=131001, hi=131001,
             heads=32, kv_heads=4, dim=128, window=0),
        # the widest batch of the long page
        dict(name="attend 64 x 8192", op="attend", dtype="fp16", seqs=64, lo=8192, hi=8192,
             heads=16, kv_heads=8, dim=64, window=0),
        # one row of the smaller vocabulary, common chat settings
        dict(name="sample one row", op="sample", dtype="fp16", rows=1, vocab=4096, kind="both"),
        # the serving batch's rows, each with settings of its own
        dict(name="sample 32 rows", op="sample", dtype="fp32", rows=32, vocab=59392, kind="mixed"),
        # every row of a serving window
        dict(name="sample 544 rows", op="sample", dtype="bf16", rows=544, vocab=59392, kind="top_p"),
        # eight forks of a sequence: the page that they go on writing, all 24 layers
        dict(name="copy 8 forks", op="copy", dtype="fp16", pages=8, layers=24, kv_heads=8, dim=64,
             shared=True),
        # closing the gaps of a pool after long sequences have left it
        dict(name="copy 900 pages", op="copy", dtype="bf16", pages=900, layers=4, kv_heads=8,
             dim=128, shared=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("append", "attend", "sample", "copy"))
    if op == "append":
        dim = rng.choice((64, 128))
        kv_heads = rng.choice((1, 2, 4, 8))
        heads = kv_heads * rng.choice((1, 2, 4, 5, 8))
        if rng.random() < 0.5:
            seqs = _log_int(rng, 1, 256)
            tokens = seqs
        else:
            tokens = _log_int(rng, 2, 8000) | 1
            seqs = rng.randint(1, min(8, tokens))
        return dict(op="append", dtype=rng.choice(("fp16", "bf16")), tokens=tokens, seqs=seqs,
                    first=rng.randint(0, 400), heads=min(heads, 32), kv_heads=kv_heads, dim=dim,
                    rot=rng.choice((16, 32, 48, 64, dim)), layout=rng.choice(("half", "interleaved")),
                    norm=rng.random() < 0.7)
    if op == "attend":
        dim = rng.choice((64, 128))
        kv_heads = rng.choice((1, 2, 4, 8))
        group = rng.choice((1, 2, 3, 4, 7, 8, 12, 16, 24))
        seqs = _log_int(rng, 1, 64)
        most = (64 * 8192 * 8 * 64) // (seqs * kv_heads * dim)       # no more than the largest
        hi = _log_int(rng, 1, min(131072, most)) | 1
        hi = min(hi, most)
        lo = rng.choice((0, hi // 4, hi))
        window = rng.choice((0, 0, 0, max(1, hi // 3) | 1))
        return dict(op="attend", dtype=rng.choice(("fp16", "bf16")), seqs=seqs, lo=lo, hi=hi,
                    heads=kv_heads * group, kv_heads=kv_heads, dim=dim, window=window)
    if op == "sample":
        return dict(op="sample", dtype=rng.choice(("fp16", "bf16", "fp32")),
                    rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 1000, 120000) | 1,
                    kind=rng.choice(("plain", "top_k", "top_p", "min_p", "both", "mixed")))
    return dict(op="copy", dtype=rng.choice(("fp16", "bf16")), pages=_log_int(rng, 1, 700),
                layers=rng.randint(1, 4), kv_heads=rng.choice((1, 2, 4, 8)),
                dim=rng.choice((64, 128)), shared=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 31))


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def _perm(g, n, count=None):
    return torch.randperm(n, device="cuda", generator=g)[:count].to(torch.int32)


def _pool(g, pages, kv_heads, dim, dtype):
    """A pool whose pages hold what earlier tokens left there."""
    pool = torch.empty(pages, 2, kv_heads, PAGE * dim, dtype=dtype, device="cuda")
    return pool.normal_(generator=g)


def _lengths(case):
    """Evenly spread lengths: their total is the case's, their order the seed's."""
    b = torch.arange(case["seqs"], dtype=torch.float64)
    top = max(1, case["seqs"] - 1)
    return (case["lo"] + torch.round((case["hi"] - case["lo"]) * b / top).to(torch.int64)
            if case["seqs"] > 1 else torch.tensor([case["hi"]]))


def _append_runs(case):
    """(sequence, slot) of every token: equal runs, each starting at its own slot."""
    t, s = case["tokens"], case["seqs"]
    seq = torch.arange(t, dtype=torch.int64) * s // t
    start = torch.searchsorted(seq, torch.arange(s))
    slot = case["first"] + 3 * seq % 61 + torch.arange(t) - start[seq]
    return seq, slot


def _rotation_angles(case, rows):
    """Angles in 64 bits: base 10000, positions stretched by 4 as for a longer context."""
    half = case["rot"] // 2
    inv = 10000.0 ** (-torch.arange(half, dtype=torch.float64) * 2.0 / case["rot"])
    return (torch.arange(rows, dtype=torch.float64) / 4.0)[:, None] * inv[None, :]


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": dict(case), "op": op}
    dt = DTYPES[case["dtype"]]
    if op == "append":
        hq, hkv, d, t = case["heads"], case["kv_heads"], case["dim"], case["tokens"]
        seq, slot = _append_runs(case)
        per = int(slot.max()) // PAGE + 1
        pages = case["seqs"] * per + 3
        angle = _rotation_angles(case, int(slot.max()) + 1)
        s.update(
            qkv=_randn(g, t, (hq + 2 * hkv) * d, dtype=dt),
            q_gain=(1 + 0.1 * _randn(g, d)).to(torch.bfloat16) if case["norm"] else None,
            k_gain=(1 + 0.1 * _randn(g, d)).to(torch.bfloat16) if case["norm"] else None,
            rope=torch.stack([angle.cos(), angle.sin()], dim=-1).float().cuda(),
            pool=_pool(g, pages, hkv, d, dt),
            pages=_perm(g, pages, case["seqs"] * per).view(case["seqs"], per),
            seq=seq.to(torch.int32).cuda(), slot=slot.to(torch.int32).cuda(),
            q=torch.zeros(t, hq, d, dtype=dt, device="cuda"),
            err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    elif op == "attend":
        hq, hkv, d, b = case["heads"], case["kv_heads"], case["dim"], case["seqs"]
        order = torch.randperm(b, device="cuda", generator=g)
        n = _lengths(case).cuda()[order]
        per = max(1, -(-case["hi"] // PAGE))
        pages = b * per + 5
        s.update(
            q=_randn(g, b, hq, d, dtype=dt, scale=2.0),
            pool=_pool(g, pages, hkv, d, dt),
            pages=_perm(g, pages, b * per).view(b, per), n=n.to(torch.int32),
            out=torch.zeros(b, hq, d, dtype=dt, device="cuda"),
            lse=torch.zeros(b, hq, device="cuda"), scratch=None)
    elif op == "sample":
        r, v = case["rows"], case["vocab"]
        x = _randn(g, r, v, scale=2.5)
        at = torch.randint(0, v, (r, 8), device="cuda", generator=g)      # what the context favours
        x.scatter_add_(1, at, 3 + 9 * torch.rand(r, 8, device="cuda", generator=g))
        x[:, v - 1] = NEG_INF                                             # never sampled: the mask token
        kind = case["kind"]
        i = torch.arange(r, device="cuda")

        def of(values, on):
            t = torch.tensor(values, device="cuda")
            return t[(i + seed) % len(values)] if on else None
        s.update(
            logits=x.to(dt), u=torch.rand(r, device="cuda", generator=g),
            temperature=of([0.7, 1.0, 1.3, 0.0, 0.9], True) if kind == "mixed" else of([0.8], True),
            top_k=of([0, 50, 1000, 1, 20], kind == "mixed") if kind == "mixed"
            else of([50], kind in ("top_k", "both")),
            top_p=of([1.0, 0.9, 0.95, 0.5], kind == "mixed") if kind == "mixed"
            else of([0.9], kind in ("top_p", "both")),
            min_p=of([0.0, 0.05, 0.0], kind == "mixed") if kind == "mixed"
            else of([0.05], kind == "min_p"),
            token=torch.zeros(r, dtype=torch.int32, device="cuda"),
            logprob=torch.zeros(r, device="cuda"), kept=torch.zeros(r, dtype=torch.int32, device="cuda"))
        if s["top_k"] is not None:
            s["top_k"] = s["top_k"].to(torch.int32)
    else:
        m, layers = case["pages"], case["layers"]
        pages = 2 * m + 3
        ids = _perm(g, pages)
        src = ids[:1].expand(m) if case["shared"] else ids[:m]
        s.update(pool=_pool(g, layers * pages, case["kv_heads"], case["dim"], dt)
                 .view(layers, pages, -1), src=src.contiguous(), dst=ids[m:2 * m].contiguous(),
                 err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return s


# -------------------------------------------------------------- plain forms
def _plain_append(s):
    c = s["case"]
    hq, hkv, d, rot, t = c["heads"], c["kv_heads"], c["dim"], c["rot"], c["tokens"]
    x = s["qkv"].float().view(t, hq + 2 * hkv, d)
    qk, v = x[:, :hq + hkv], x[:, hq + hkv:]
    if c["norm"]:
        gain = torch.cat([s["q_gain"].float().expand(hq, d), s["k_gain"].float().expand(hkv, d)])
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + 1e-6) * gain
    cs = s["rope"][s["slot"].long()][:, None]
    cos, sin = cs[..., 0], cs[..., 1]
    if c["layout"] == "half":
        a, b = qk[..., :rot // 2], qk[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = qk[..., 0:rot:2], qk[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    qk = torch.cat([turned, qk[..., rot:]], dim=-1).to(s["qkv"].dtype)
    page = s["pages"][s["seq"].long(), s["slot"].long() // PAGE].long()
    at = s["slot"].long() % PAGE
    pool = s["pool"]
    pool.view(-1, 2, hkv, PAGE, d)[page, 0, :, at] = qk[:, hq:]
    pool.view(-1, 2, hkv, d, PAGE)[page, 1, :, :, at] = v.to(pool.dtype)
    s["q"].copy_(qk[:, :hq])
    return {"q": s["q"], "pool": pool}


def _plain_attend(s):
    c = s["case"]
    hq, hkv, d, b = c["heads"], c["kv_heads"], c["dim"], c["seqs"]
    per = s["pages"].shape[1]
    kv = s["pool"][s["pages"].long()]                                  # [b, per, 2, hkv, 64 * d]
    k = kv[:, :, 0].view(b, per, hkv, PAGE, d).permute(0, 2, 4, 1, 3).float().reshape(b, hkv, d, -1)
    v = kv[:, :, 1].view(b, per, hkv, d, PAGE).permute(0, 2, 1, 4, 3).float().reshape(b, hkv, -1, d)
    q = s["q"].float().view(b, hkv, hq // hkv, d)
    score = torch.matmul(q, k) * (d ** -0.5)
    at = torch.arange(per * PAGE, device=score.device)
    n = s["n"].long()[:, None]
    seen = at < n
    if c["window"]:
        seen = seen & (at >= n - c["window"])
    seen = seen[:, None, None, :]
    score = score.masked_fill(~seen, NEG_INF)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    # a value behind the mask may hold anything: it counts for nothing
    v = torch.where(seen.transpose(-1, -2), v, 0.0)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(out.view(b, hq, d))
    s["lse"].copy_((torch.log(total) + top).view(b, hq))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_sample(s):
    x = s["logits"].float() + 0.0
    x = torch.where(torch.isnan(x), NEG_INF, x)
    x, order = torch.sort(x, dim=-1, descending=True, stable=True)      # ties: the lowest index
    rows, v = x.shape
    top = x[:, :1]
    t = s["temperature"][:, None]
    d = torch.where(x == top, 0.0, (x - top) * (1.0 / t))
    w = torch.where((x == NEG_INF), 0.0, torch.exp(d))
    mass = (w * MASS_ONE).to(torch.int64)
    at = torch.arange(v, device=x.device)
    kept = mass > 0
    if s["min_p"] is not None:
        kept &= w >= s["min_p"][:, None].clamp(max=1.0)
    if s["top_k"] is not None:
        k = s["top_k"][:, None].long()
        kept &= (at < k) | (k <= 0)
    kept &= (at == 0) | (t > 0)                                         # no temperature: the best one
    mass = torch.where(kept, mass, 0)
    cum = mass.cumsum(-1)
    if s["top_p"] is not None:
        p = s["top_p"][:, None].double()
        need = torch.ceil(p * cum[:, -1:].double()).long().clamp(min=1)
        kept &= (cum - mass < need) | (p >= 1)
        mass = torch.where(kept, mass, 0)
        cum = mass.cumsum(-1)
    total = cum[:, -1:]
    r = torch.minimum((s["u"][:, None].double() * total.double()).long(), total - 1)
    hit = (cum > r).int().argmax(-1, keepdim=True)
    any_left = top > NEG_INF
    share = mass.gather(1, hit).double() / total.double()
    s["token"].copy_(torch.where(any_left, order.gather(1, hit), -1)[:, 0])
    s["logprob"].copy_(torch.where(any_left, torch.log(share), NEG_INF)[:, 0])
    s["kept"].copy_((kept & any_left).sum(-1))
    return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}


def _plain_copy(s):
    s["pool"][:, s["dst"].long()] = s["pool"][:, s["src"].long()]
    return s["pool"]


# ------------------------------------------------- the framework's operators
def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _cache(s, gs):
    """The descriptors that a program makes once for its cache."""
    c = s["case"]
    dt = {"fp16": gs.GS_F16, "bf16": gs.GS_BF16}[c["dtype"]]
    s["cache"] = gs.gs_cache(s["pool"].data_ptr(), s["pool"].shape[0], c["kv_heads"], c["dim"], dt,
                             s["pages"].data_ptr(), s["pages"].shape[0], s["pages"].shape[1])
    return s["cache"]


def _own_append(s, gs):
    c = s["case"]
    cache = s.get("cache") or _cache(s, gs)
    if "turn" not in s:
        layout = gs.ROPE_HALF if c["layout"] == "half" else gs.ROPE_INTERLEAVED
        s["turn"] = gs.gs_rope(s["rope"].data_ptr(), s["rope"].shape[0], c["rot"], layout)
    gs.gs_rope_append(cache, s["turn"], s["qkv"].data_ptr(), s["qkv"].shape[1], c["tokens"],
                      c["heads"], _ptr(s["q_gain"]), _ptr(s["k_gain"]), 1e-6, s["seq"].data_ptr(),
                      s["slot"].data_ptr(), s["slot"].data_ptr(), s["q"].data_ptr(),
                      c["heads"] * c["dim"], s["err"].data_ptr(),
                      torch.cuda.current_stream().cuda_stream)
    return {"q": s["q"], "pool": s["pool"]}


def _own_attend(s, gs):
    c = s["case"]
    cache = s.get("cache") or _cache(s, gs)
    if s["scratch"] is None:
        s["scratch"] = torch.zeros(gs.gs_decode_attention_scratch_bytes(
            cache, c["seqs"], c["heads"], 0), dtype=torch.uint8, device="cuda")
    hd = c["heads"] * c["dim"]
    gs.gs_decode_attention(cache, s["q"].data_ptr(), hd, 0, s["n"].data_ptr(), c["seqs"],
                           c["heads"], c["dim"] ** -0.5, c["window"], s["out"].data_ptr(), hd,
                           s["lse"].data_ptr(), 0, s["scratch"].data_ptr(), s["scratch"].numel(),
                           torch.cuda.current_stream().cuda_stream)
    return {"out": s["out"], "lse": s["lse"]}


def _own_sample(s, gs):
    if "params" not in s:
        s["params"] = gs.gs_sample_params(_ptr(s["temperature"]), _ptr(s["top_p"]),
                                          _ptr(s["min_p"]), _ptr(s["top_k"]))
    x = s["logits"]
    dt = {torch.float16: gs.GS_F16, torch.bfloat16: gs.GS_BF16, torch.float32: gs.GS_F32}[x.dtype]
    gs.gs_sample(x.data_ptr(), x.shape[1], x.shape[0], x.shape[1], dt, s["params"],
                 s["u"].data_ptr(), s["token"].data_ptr(), s["logprob"].data_ptr(),
                 s["kept"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return {"token": s["token"], "logprob": s["logprob"], "kept": s["kept"]}


def _own_copy(s, gs):
    pool = s["pool"]
    layers, pages, elems = pool.shape
    gs.gs_pages_copy(pool.data_ptr(), pages, pool.data_ptr(), pages, layers, elems * 2,
                     s["src"].data_ptr(), s["dst"].data_ptr(), s["src"].shape[0],
                     s["err"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    return pool


def run(state):
    op = state["op"]
    if own:
        from paper_2609_26638_gb300 import gs
        return {"append": _own_append, "attend": _own_attend, "sample": _own_sample,
                "copy": _own_copy}[op](state, gs)
    return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample,
            "copy": _plain_copy}[op](state)


def work(case):
    op = case["op"]
    if op == "append":
        t, d = case["tokens"], case["dim"]
        heads = case["heads"] + 2 * case["kv_heads"]
        rows = t if case["seqs"] == t else int(_append_runs(case)[1].unique().numel())
        # the projected row in, queries and cache rows out, the rotation's rows, the ids
        return {"bytes": 2 * t * heads * d * 2 + rows * case["rot"] * 4 + t * 8, "flops": 8 * t * heads * d}
    if op == "attend":
        n = _lengths(case)
        seen = int((n.clamp(max=case["window"]) if case["window"] else n).sum())
        b, hq, hkv, d = case["seqs"], case["heads"], case["kv_heads"], case["dim"]
        return {"bytes": seen * hkv * d * 4 + b * hq * (d * 4 + 4) + 4 * b + seen // 16,
                "flops": 4 * seen * hq * d}
    if op == "sample":
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": case["rows"] * (case["vocab"] * size + 32),
                "flops": 8 * case["rows"] * case["vocab"]}
    page = case["layers"] * 2 * case["kv_heads"] * PAGE * case["dim"] * 2
    reads = 1 if case["shared"] else case["pages"]
    return {"bytes": (reads + case["pages"]) * page + 8 * case["pages"], "flops": 0}


# ----------------------------------------------------------------- 64 bits
def _exact_append(case, s):
    hq, hkv, d, t = case["heads"], case["kv_heads"], case["dim"], case["tokens"]
    x = s["qkv"].cpu().double().numpy().reshape(t, hq + 2 * hkv, d)
    slot, seq = s["slot"].cpu().numpy(), s["seq"].cpu().numpy()
    y = x[:, :hq + hkv].copy()
    if case["norm"]:
        y /= np.sqrt((y * y).sum(-1, keepdims=True) / d + 1e-6)
        y[:, :hq] *= s["q_gain"].cpu().double().numpy()
        y[:, hq:] *= s["k_gain"].cpu().double().numpy()
    angle = _rotation_angles(case, int(slot.max()) + 1).numpy()[slot][:, None]
    half = case["rot"] // 2
    i = np.arange(half)
    first, second = (i, i + half) if case["layout"] == "half" else (2 * i, 2 * i + 1)
    z = (y[..., first] + 1j * y[..., second]) * np.exp(1j * angle)
    y[..., first], y[..., second] = z.real, z.imag
    pool = s["pool"].cpu().double().numpy()
    page = s["pages"].cpu().numpy()[seq, slot // PAGE]
    pool.reshape(-1, 2, hkv, PAGE, d)[page, 0, :, slot % PAGE] = y[:, hq:]
    pool.reshape(-1, 2, hkv, d, PAGE)[page, 1, :, :, slot % PAGE] = x[:, hq + hkv:]
    return {"q": y[:, :hq], "pool": pool}


def _exact_attend(case, s):
    hq, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(case["seqs"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((case["seqs"], hq), NEG_INF, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["n"].tolist()):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n - first < 1:
            continue
        used = s["pages"][b, :-(-n // PAGE)].long()
        kv = s["pool"][used].double()
        k = kv[:, 0].view(-1, hkv, PAGE, d).transpose(0, 1).reshape(hkv, -1, d)[:, first:n]
        v = kv[:, 1].view(-1, hkv, d, PAGE).permute(1, 0, 3, 2).reshape(hkv, -1, d)[:, first:n]
        q = s["q"][b].double().view(hkv, hq // hkv, d)
        z = torch.einsum("hgd,hnd->hgn", q, k) / np.sqrt(d)
        lse[b] = torch.logsumexp(z, -1).view(hq)
        out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(z, -1), v).reshape(hq, d)
    return {"out": out.cpu().numpy(), "lse": lse.cpu().numpy()}


def _exact_sample(case, s):
    x = s["logits"].cpu().double().numpy()
    u = s["u"].cpu().double().numpy()
    par = {k: None if s[k] is None else s[k].cpu().double().numpy()
           for k in ("temperature", "top_k", "top_p", "min_p")}
    logprob = np.zeros(len(x))
    for i, row in enumerate(x):
        t = par["temperature"][i]
        if t <= 0:
            continue                                      # the best token, with certainty
        order = np.argsort(-row, kind="stable")
        w = np.exp((row[order] - row[order[0]]) / t)
        if par["min_p"] is not None:
            w = w[w >= par["min_p"][i]]
        if par["top_k"] is not None and par["top_k"][i] > 0:
            w = w[:int(par["top_k"][i])]
        if par["top_p"] is not None and par["top_p"][i] < 1:
            w = w[:int(np.searchsorted(w.cumsum(), par["top_p"][i] * w.sum())) + 1]
        share = w / w.sum()
        at = min(int(np.searchsorted(share.cumsum(), u[i], side="right")), len(w) - 1)
        logprob[i] = np.log(share[at])
    return {"token": None, "logprob": logprob, "kept": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, s)
    if case["op"] == "attend":
        return _exact_attend(case, s)
    if case["op"] == "sample":
        return _exact_sample(case, s)
    pool = s["pool"].clone()                              # copies are exact in any type
    for src, dst in zip(s["src"].tolist(), s["dst"].tolist()):
        pool[:, dst] = s["pool"][:, src]
    return pool
