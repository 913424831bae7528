"""Cases and plain forms of the operators that verify a tree of drafted tokens.

Four operators make one verifying step of a decoder over a paged key-value
cache, when several tokens are drafted ahead as a tree of candidates:

  attend  attention of every node of the tree: the cached tokens, and of the
          tree the nodes that a 64-bit mask names (its ancestors and itself)
  accept  the path from the root along the nodes that carry the token which the
          model chose at their parent
  commit  keys and values of that path moved to consecutive slots, all layers
  w4      products with 4-bit weights and group scales, for the few rows that a
          step has

Node i of a tree lies in the cache at slot n + i until it is accepted.  A page
holds 64 tokens of one layer: [2][kv heads][64 * head_dim], keys as [64
tokens][head_dim], values transposed as [head_dim][64 tokens].
"""
import numpy as np
import torch

own = False

PAGE = 64
VOCAB = 59392
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
NEG_INF = float("-inf")


# ------------------------------------------------------------------- cases
def listed():
    return [
        # a chain of four tokens after the last one, short context: latency
        dict(name="attend chain short", op="attend", dtype="fp16", seqs=1, lo=517, hi=517, nodes=5,
             heads=16, kv_heads=8, dim=64, window=0, ragged=False),
        # the serving batch: 32 sequences of 1024 to 6144 tokens, 16 drafted nodes each
        dict(name="attend serving 32 x 17", op="attend", dtype="fp16", seqs=32, lo=1024, hi=6144,
             nodes=17, heads=16, kv_heads=8, dim=64, window=0, ragged=True),
        # one very long document and a wide tree
        dict(name="attend long x 33", op="attend", dtype="bf16", seqs=1, lo=65001, hi=65001, nodes=33,
             heads=32, kv_heads=4, dim=128, window=0, ragged=False),
        # the widest batch of the long page, a short chain
        dict(name="attend 64 x 8192 x 8", op="attend", dtype="fp16", seqs=64, lo=8192, hi=8192,
             nodes=8, heads=16, kv_heads=8, dim=64, window=0, ragged=False),
        # one sequence's step
        dict(name="accept one tree", op="accept", trees=1, chains=4, depth=4, shape="chains"),
        # every sequence of a large batch, the widest trees
        dict(name="accept 256 x 64", op="accept", trees=256, chains=7, depth=9, shape="random"),
        # one sequence: all 24 layers
        dict(name="commit one", op="commit", dtype="fp16", trees=1, chains=4, depth=4, layers=24,
             kv_heads=8, dim=64, lo=2048, hi=2048),
        # a batch of long chains with wide heads
        dict(name="commit 64", op="commit", dtype="bf16", trees=64, chains=3, depth=16, layers=12,
             kv_heads=8, dim=128, lo=100, hi=700),
        # the output projection of one sequence's next token: latency
        dict(name="w4 one row", op="w4", dtype="fp16", rows=1, out=1024, inner=1024, group=64,
             zeros=False, gated=False),
        # gate and up of one sequence's tree
        dict(name="w4 gate/up 17 rows", op="w4", dtype="fp16", rows=17, out=4096, inner=1024,
             group=32, zeros=True, gated=True),
        # the vocabulary's logits for a short chain
        dict(name="w4 vocabulary 5 rows", op="w4", dtype="bf16", rows=5, out=VOCAB, inner=1024,
             group=128, zeros=False, gated=False),
        # a wide layer, the serving batch's next tokens
        dict(name="w4 wide 32 rows", op="w4", dtype="bf16", rows=32, out=8192, inner=8192, group=128,
             zeros=True, gated=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("attend", "attend", "accept", "commit", "w4", "w4"))
    if op == "attend":
        dim = rng.choice((64, 128))
        kv_heads = rng.choice((1, 2, 4, 8))
        group = rng.choice((1, 2, 3, 4, 5, 8))
        nodes = _log_int(rng, 1, 64)
        seqs = _log_int(rng, 1, 64)
        # no more bytes, and no more arithmetic, than the largest
        most = min(64 * 8192 * 8 * 64 // (seqs * kv_heads * dim),
                   4 * 10 ** 10 // (4 * seqs * kv_heads * group * dim * nodes))
        hi = min(_log_int(rng, 1, max(2, min(131072, most))) | 1, max(1, most))
        return dict(op="attend", dtype=rng.choice(("fp16", "bf16")), seqs=seqs,
                    lo=rng.choice((0, hi // 4, hi)), hi=hi, nodes=nodes, heads=kv_heads * group,
                    kv_heads=kv_heads, dim=dim, window=rng.choice((0, 0, 0, max(1, hi // 3) | 1)),
                    ragged=rng.random() < 0.5)
    chains, depth = rng.randint(1, 8), rng.randint(1, 7)
    if op == "accept":
        return dict(op="accept", trees=_log_int(rng, 1, 400), chains=chains, depth=depth,
                    shape=rng.choice(("chains", "random")))
    if op == "commit":
        hi = _log_int(rng, 1, 700)
        return dict(op="commit", dtype=rng.choice(("fp16", "bf16")), trees=_log_int(rng, 1, 48),
                    chains=chains, depth=depth, layers=rng.randint(1, 12),
                    kv_heads=rng.choice((1, 2, 4, 8)), dim=rng.choice((64, 128)),
                    lo=rng.choice((0, hi // 2, hi)), hi=hi)
    group = rng.choice((32, 64, 128))
    gated = rng.random() < 0.3
    inner = group * max(1, _log_int(rng, 64, 8192) // group)
    out = _log_int(rng, 40, min(60000, 8192 * 8192 // inner) // (2 if gated else 1))
    return dict(op="w4", dtype=rng.choice(("fp16", "bf16")), rows=_log_int(rng, 1, 64 if out * inner < 2 ** 24 else 16),
                out=max(8, out // 8 * 8) if gated else out, inner=inner, group=group,
                zeros=rng.random() < 0.5, gated=gated)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 31))


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def _lengths(case, count):
    """Evenly spread lengths: their total is the case's, their order the seed's."""
    b = np.arange(count, dtype=np.float64) / max(1, count - 1)
    return np.array([case["hi"]]) if count == 1 else \
        (case["lo"] + np.round((case["hi"] - case["lo"]) * b)).astype(np.int64)


def _counts(case):
    """Nodes of each tree: all of them, or between half and all."""
    nodes, b = case["nodes"], np.arange(case["seqs"])
    return nodes - (b * 7919 % (nodes // 2 + 1) if case["ragged"] else 0 * b)


def _chains(trees, chains, depth):
    """Candidate continuations side by side: node 1 + c * depth + i is the i-th token of chain c."""
    i = np.arange(chains * depth)
    row = np.concatenate([[-1], np.where(i % depth == 0, 0, i)])
    return np.tile(row, (trees, 1))


def _grown(rng, trees, nodes):
    """Each node hangs on any earlier one, rather a late one."""
    i = np.arange(nodes)
    up = np.floor(i * rng.random((trees, nodes)) ** 0.5).astype(np.int64)
    up[:, 0] = -1
    return up


def _masks(parent):
    """Ancestors and the node itself, as bits; and the node's depth."""
    trees, nodes = parent.shape
    mask, depth = np.zeros((trees, nodes), np.uint64), np.zeros((trees, nodes), np.int64)
    for i in range(nodes):
        mask[:, i] = np.uint64(1 << i)
        if i:
            at = parent[:, i: i + 1]
            mask[:, i] |= np.take_along_axis(mask, at, 1)[:, 0]
            depth[:, i] = 1 + np.take_along_axis(depth, at, 1)[:, 0]
    return mask, depth


def _cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _paged(s, g, case, count, slots, layers=1):
    """A pool whose pages hold what earlier tokens left there, in shuffled order."""
    per = max(1, -(-int(slots) // PAGE))
    pages = count * per + 5
    s["pool"] = torch.empty(layers, pages, 2, case["kv_heads"], PAGE * case["dim"],
                            dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g)
    s["pages"] = torch.randperm(pages, device="cuda", generator=g)[: count * per].to(
        torch.int32).view(count, per)


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    op = case["op"]
    s = {"case": dict(case), "op": op}
    if op == "attend":
        b, t, hq, d = case["seqs"], case["nodes"], case["heads"], case["dim"]
        parent = _grown(rng, b, t)
        mask, depth = _masks(parent)
        n = rng.permutation(_lengths(case, b))
        _paged(s, g, case, b, int(n.max()) + t)
        s.update(q=_randn(g, b * t, hq * d, dtype=DTYPES[case["dtype"]], scale=2.0), n=_cuda(n),
                 mask=_cuda(mask.view(np.int64), torch.int64), pos=_cuda(n[:, None] + depth),
                 count=_cuda(_counts(case)) if case["ragged"] else None,
                 out=torch.zeros(b * t, hq * d, dtype=DTYPES[case["dtype"]], device="cuda"),
                 lse=torch.zeros(b * t, hq, device="cuda"), scratch=None)
    elif op == "accept":
        b, t = case["trees"], 1 + case["chains"] * case["depth"]
        parent = _chains(b, case["chains"], case["depth"]) if case["shape"] == "chains" \
            else _grown(rng, b, t)
        token = rng.integers(0, VOCAB, (b, t))
        choice = rng.integers(0, VOCAB, (b, t))
        for i in range(t - 1, 0, -1):              # most nodes' choices are drafted at one child
            hit = rng.random(b) < 0.7
            np.put_along_axis(choice, parent[:, i: i + 1],
                              np.where(hit, token[:, i],
                                       np.take_along_axis(choice, parent[:, i: i + 1], 1)[:, 0])[:, None], 1)
        s.update(parent=_cuda(parent), token=_cuda(token), choice=_cuda(choice),
                 path=torch.zeros(b, t, dtype=torch.int32, device="cuda"),
                 new=torch.zeros(b, t, dtype=torch.int32, device="cuda"),
                 length=torch.zeros(b, dtype=torch.int32, device="cuda"),
                 err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    elif op == "commit":
        b, t = case["trees"], 1 + case["chains"] * case["depth"]
        n = rng.permutation(_lengths(case, b))
        _paged(s, g, case, b, int(n.max()) + t, case["layers"])
        path, length = _paths(case, rng)
        s.update(n=_cuda(n), path=_cuda(path), length=_cuda(length),
                 err=torch.zeros(1, dtype=torch.int32, device="cuda"))
    else:
        dt, m, k = DTYPES[case["dtype"]], case["rows"], case["inner"]
        rows = case["out"] * (2 if case["gated"] else 1)
        q = (_randn(g, rows, k, scale=3.0) + 8).round().clamp(0, 15).to(torch.uint8)
        s.update(x=_randn(g, m, k, dtype=dt),
                 q=q[:, 0::2] | (q[:, 1::2] << 4),
                 scale=(0.01 * (1 + 0.3 * torch.rand(rows, k // case["group"], device="cuda",
                                                     generator=g))).to(dt),
                 zero=torch.randint(5, 12, (rows, k // case["group"]), device="cuda", generator=g,
                                    dtype=torch.uint8) if case["zeros"] else None,
                 y=torch.zeros(m, case["out"], dtype=dt, device="cuda"),
                 err=torch.zeros(1, dtype=torch.int32, device="cuda"))
        if own:                                    # laid out once, as a decoder's weights are
            _pack(s)
    return s


def _paths(case, rng):
    """Accepted paths: how many tokens is the tree's number's, which chain the seed's."""
    b, depth = np.arange(case["trees"]), case["depth"]
    length = 1 + (b * 5 + depth - 1) % (depth + 1) if case["trees"] > 1 else np.array([depth + 1])
    chain = rng.integers(min(1, case["chains"] - 1), case["chains"], case["trees"])
    i = np.arange(1 + case["chains"] * depth)
    path = np.where(i == 0, 0, chain[:, None] * depth + i)
    return np.where(i < length[:, None], path, -1), length


# -------------------------------------------------------------- plain forms
def _plain_attend(s):
    c = s["case"]
    hq, hkv, d, b, t = c["heads"], c["kv_heads"], c["dim"], c["seqs"], c["nodes"]
    per = s["pages"].shape[1]
    kv = s["pool"][0][s["pages"].long()]                               # [b, per, 2, hkv, 64 * d]
    k = kv[:, :, 0].view(b, per, hkv, PAGE, d).permute(0, 2, 4, 1, 3).float().reshape(b, hkv, d, -1)
    v = kv[:, :, 1].view(b, per, hkv, d, PAGE).permute(0, 2, 1, 4, 3).float().reshape(b, hkv, -1, d)
    q = s["q"].float().view(b, t, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, d)
    score = (torch.matmul(q, k) * (d ** -0.5)).view(b, hkv, hq // hkv, t, -1)
    n, at = s["n"].long()[:, None, None], torch.arange(per * PAGE, device=q.device)
    count = s["count"].long()[:, None, None] if c["ragged"] else torch.full_like(n, t)
    node = at - n                                                      # [b, 1, slots]
    seen = (s["mask"][:, :, None] >> node.clamp(0, 63)) & 1            # [b, t, slots]
    seen = torch.where(node < 0, 1, seen) * (node < count)
    if c["window"]:
        seen = seen * ((at > s["pos"].long()[:, :, None] - c["window"]) | (node >= 0))
    seen = (seen > 0)[:, None, None]
    score = score.masked_fill(~seen, NEG_INF)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, hkv, -1, per * PAGE), v).view(b, hkv, hq // hkv, t, d)
    out = (out / torch.where(total > 0, total, 1.0)).permute(0, 3, 1, 2, 4)
    lse = (torch.log(total) + top)[..., 0].permute(0, 3, 1, 2)
    used = (torch.arange(t, device=q.device) < count[:, 0])[:, :, None]
    s["out"].copy_(torch.where(used, out.reshape(b, t, -1), s["out"].view(b, t, -1)).reshape(b * t, -1))
    s["lse"].copy_(torch.where(used, lse.reshape(b, t, -1), s["lse"].view(b, t, -1)).reshape(b * t, -1))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_accept(s):
    parent, token, choice = s["parent"].long(), s["token"], s["choice"]
    b, t = parent.shape
    node = torch.arange(t, device=parent.device)
    match = (token == choice.gather(1, parent.clamp(min=0))) & (node > 0)
    cur = torch.zeros(b, 1, dtype=torch.int64, device=parent.device)
    live = torch.ones(b, 1, dtype=torch.bool, device=parent.device)
    s["length"].zero_()
    for i in range(t):
        s["path"][:, i: i + 1] = torch.where(live, cur, -1).int()
        s["new"][:, i: i + 1] = torch.where(live, choice.gather(1, cur), -1)
        s["length"] += live[:, 0]
        child = match & (parent == cur)
        live = live & child.any(1, keepdim=True)
        cur = child.int().argmax(1, keepdim=True)                      # the lowest index
    return {"path": s["path"], "new": s["new"], "length": s["length"]}


def _plain_commit(s):
    c, pool = s["case"], s["pool"]
    layers, pages, _, hkv, _ = pool.shape
    i = torch.arange(s["path"].shape[1], device=pool.device)
    tree, i = torch.nonzero(i < s["length"][:, None], as_tuple=True)
    src = s["n"].long()[tree] + s["path"].long()[tree, i]
    dst = s["n"].long()[tree] + i
    at = s["pages"].long()
    src, src_page = src % PAGE, at[tree, src // PAGE]
    dst, dst_page = dst % PAGE, at[tree, dst // PAGE]
    k = pool.view(layers, pages, 2, hkv, PAGE, c["dim"])
    v = pool.view(layers, pages, 2, hkv, c["dim"], PAGE)
    k[:, dst_page, 0, :, dst] = k[:, src_page, 0, :, src]
    v[:, dst_page, 1, :, :, dst] = v[:, src_page, 1, :, :, src]
    return pool


def _weights(s, dtype):
    c = s["case"]
    q = torch.stack([s["q"] & 15, s["q"] >> 4], dim=-1).flatten(1).to(dtype)
    zero = 8.0 if s["zero"] is None else s["zero"].to(dtype).repeat_interleave(c["group"], 1)
    return (q - zero) * s["scale"].to(dtype).repeat_interleave(c["group"], 1)


def _plain_w4(s):
    y = torch.matmul(s["x"].float(), _weights(s, torch.float32).t())
    if s["case"]["gated"]:
        gate, up = y.chunk(2, dim=-1)
        y = gate / (1 + torch.exp(-gate)) * up
    s["y"].copy_(y)
    return s["y"]


# ------------------------------------------------- the framework's operators
def _ptr(t):
    return t.data_ptr() if t is not None else 0


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _dtype(gs, case):
    return {"fp16": gs.GS_F16, "bf16": gs.GS_BF16}[case["dtype"]]


def _cache(s, gs):
    """The descriptor that a program makes once for its cache."""
    c = s["case"]
    if "cache" not in s:
        s["cache"] = gs.gs_cache(s["pool"].data_ptr(), s["pool"].shape[1], c["kv_heads"], c["dim"],
                                 _dtype(gs, c), s["pages"].data_ptr(), s["pages"].shape[0],
                                 s["pages"].shape[1])
    return s["cache"]


def _own_attend(s, gs):
    c = s["case"]
    cache = _cache(s, gs)
    if s["scratch"] is None:
        s["scratch"] = torch.zeros(gs.gs_tree_attention_scratch_bytes(
            cache, c["seqs"], c["nodes"], c["heads"], 0), dtype=torch.uint8, device="cuda")
    hd = c["heads"] * c["dim"]
    gs.gs_tree_attention(cache, s["q"].data_ptr(), hd, 0, s["n"].data_ptr(), _ptr(s["count"]),
                         s["mask"].data_ptr(), s["pos"].data_ptr(), c["seqs"], c["nodes"], c["heads"],
                         c["dim"] ** -0.5, c["window"], s["out"].data_ptr(), hd, s["lse"].data_ptr(),
                         0, s["scratch"].data_ptr(), s["scratch"].numel(), _stream())
    return {"out": s["out"], "lse": s["lse"]}


def _own_accept(s, gs):
    trees, nodes = s["parent"].shape
    gs.gs_tree_accept(s["parent"].data_ptr(), s["token"].data_ptr(), s["choice"].data_ptr(), 0, 0, -1,
                      trees, nodes, s["path"].data_ptr(), s["new"].data_ptr(), s["length"].data_ptr(),
                      s["err"].data_ptr(), _stream())
    return {"path": s["path"], "new": s["new"], "length": s["length"]}


def _own_commit(s, gs):
    trees, nodes = s["path"].shape
    gs.gs_tree_commit(_cache(s, gs), s["pool"].shape[0], 0, s["n"].data_ptr(), s["path"].data_ptr(),
                      s["length"].data_ptr(), trees, nodes, s["err"].data_ptr(), _stream())
    return s["pool"]


def _pack(s):
    from paper_2609_26638_gb300 import gs
    c = s["case"]
    w = gs.gs_qweight(0, s["q"].shape[0], c["inner"], c["group"], _dtype(gs, c), int(c["zeros"]),
                      int(c["gated"]))
    s["packed"] = torch.empty(gs.gs_qweight_bytes(w), dtype=torch.uint8, device="cuda")
    w.packed = s["packed"].data_ptr()
    gs.gs_qweight_pack(w, s["q"].data_ptr(), s["scale"].data_ptr(), _ptr(s["zero"]), _stream())
    s["w"] = w


def _own_w4(s, gs):
    c = s["case"]
    gs.gs_qlinear(s["w"], s["x"].data_ptr(), c["inner"], s["y"].data_ptr(), c["out"], c["rows"],
                    gs.EPI_SWIGLU if c["gated"] else gs.EPI_STORE_F16, s["err"].data_ptr(), _stream())
    return s["y"]


def run(state):
    op = state["op"]
    if own:
        from paper_2609_26638_gb300 import gs
        return {"attend": _own_attend, "accept": _own_accept, "commit": _own_commit,
                "w4": _own_w4}[op](state, gs)
    return {"attend": _plain_attend, "accept": _plain_accept, "commit": _plain_commit,
            "w4": _plain_w4}[op](state)


def work(case):
    op = case["op"]
    if op == "attend":
        b, hq, hkv, d = case["seqs"], case["heads"], case["kv_heads"], case["dim"]
        n, count = _lengths(case, b), _counts(case)
        if case["window"]:
            n = np.minimum(n, case["window"] - 1)
        rows = int(count.sum())
        # K and V once, queries in and outputs out, masks, positions, the pages' numbers
        return {"bytes": int((n + count).sum()) * hkv * d * 4 + rows * (hq * (d * 4 + 4) + 12),
                "flops": 4 * int(((n + count) * count).sum()) * hq * d}
    if op == "accept":
        return {"bytes": case["trees"] * (20 * (1 + case["chains"] * case["depth"]) + 4), "flops": 0}
    if op == "commit":
        _, length = _paths(case, np.random.default_rng(0))
        moved = int((length - 1).sum()) if case["chains"] > 1 else 0
        row = case["layers"] * 2 * case["kv_heads"] * case["dim"] * 2
        return {"bytes": 2 * moved * row + int(length.sum()) * 4 + 12 * case["trees"], "flops": 0}
    rows, k, m = case["out"] * (2 if case["gated"] else 1), case["inner"], case["rows"]
    return {"bytes": rows * k // 2 + rows * k // case["group"] * (3 if case["zeros"] else 2)
            + 2 * m * (k + case["out"]), "flops": 2 * m * rows * k}


# ----------------------------------------------------------------- 64 bits
def _exact_attend(case, s):
    hq, hkv, d, t = case["heads"], case["kv_heads"], case["dim"], case["nodes"]
    out = torch.zeros(case["seqs"] * t, hq * d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["seqs"] * t, hq, dtype=torch.float64, device="cuda")
    counts = _counts(case)
    masks, pos = s["mask"].cpu().numpy().view(np.uint64), s["pos"].tolist()
    for b, n in enumerate(s["n"].tolist()):
        m = int(counts[b])
        used = s["pages"][b, : -(-(n + m) // PAGE)].long()
        kv = s["pool"][0][used].double()
        k = kv[:, 0].view(-1, hkv, PAGE, d).transpose(0, 1).reshape(hkv, -1, d)[:, : n + m]
        v = kv[:, 1].view(-1, hkv, d, PAGE).permute(1, 0, 3, 2).reshape(hkv, -1, d)[:, : n + m]
        see = np.zeros((m, n + m), bool)
        for i in range(m):
            see[i, (max(0, pos[b][i] + 1 - case["window"]) if case["window"] else 0): n] = True
            see[i, n:] = [(int(masks[b, i]) >> j) & 1 for j in range(m)]
        see = torch.from_numpy(see).cuda()
        q = s["q"].view(-1, t, hkv, hq // hkv, d)[b, :m].double()
        z = torch.einsum("thgd,hnd->thgn", q, k) / np.sqrt(d)
        z.masked_fill_(~see[:, None, None], NEG_INF)
        lse.view(-1, t, hq)[b, :m] = torch.logsumexp(z, -1).reshape(m, hq)
        out.view(-1, t, hq * d)[b, :m] = torch.einsum("thgn,hnd->thgd", torch.softmax(z, -1), v).reshape(m, -1)
    return {"out": out.cpu().numpy(), "lse": lse.cpu().numpy()}


def _exact_accept(s):
    parent, token, choice = (s[k].tolist() for k in ("parent", "token", "choice"))
    path, new, length = [], [], []
    for up, tok, want in zip(parent, token, choice):
        walk = [0]
        while True:
            nxt = [i for i in range(1, len(up)) if up[i] == walk[-1] and tok[i] == want[walk[-1]]]
            if not nxt:
                break
            walk.append(nxt[0])
        rest = [-1] * (len(up) - len(walk))
        path.append(walk + rest)
        new.append([want[i] for i in walk] + rest)
        length.append(len(walk))
    return {"path": np.array(path), "new": np.array(new), "length": np.array(length)}


def _exact_commit(case, s):
    pool = s["pool"].clone()                              # moves are exact in any type
    layers, pages, _, hkv, _ = pool.shape
    shape = {0: (layers, pages, 2, hkv, PAGE, case["dim"]), 1: (layers, pages, 2, hkv, case["dim"], PAGE)}
    table = s["pages"].tolist()
    for b, (n, path, length) in enumerate(zip(s["n"].tolist(), s["path"].tolist(), s["length"].tolist())):
        for i in range(length):
            a, z = n + path[i], n + i
            pa, pz = table[b][a // PAGE], table[b][z // PAGE]
            pool.view(shape[0])[:, pz, 0, :, z % PAGE] = s["pool"].view(shape[0])[:, pa, 0, :, a % PAGE]
            pool.view(shape[1])[:, pz, 1, :, :, z % PAGE] = s["pool"].view(shape[1])[:, pa, 1, :, :, a % PAGE]
    return pool


def _exact_w4(case, s):
    q = s["q"].to(torch.int32)
    rows, k = q.shape[0], case["inner"]
    w = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = (q % 16).double(), (q // 16).double()
    w = w.view(rows, -1, case["group"])
    w = w - (8 if s["zero"] is None else s["zero"].double()[:, :, None])
    x = s["x"].double().view(case["rows"], -1, case["group"])
    y = torch.einsum("mga,nga,ng->mn", x, w, s["scale"].double()) if rows * case["rows"] < 2 ** 10 else \
        x.flatten(1) @ (w * s["scale"].double()[:, :, None]).flatten(1).t()
    if case["gated"]:
        gate, up = y[:, : case["out"]], y[:, case["out"]:]
        y = gate * torch.sigmoid(gate) * up
    return y.cpu().numpy()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, s)
    if case["op"] == "accept":
        return _exact_accept(s)
    if case["op"] == "commit":
        return _exact_commit(case, s)
    return _exact_w4(case, s)
