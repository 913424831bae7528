"""Several sampled continuations of one prompt, token by token.

A decoder that the round engine does not cover -- RMS-normed query and key
heads, rotary positions on part of the head, 64 or 128 dims per head -- run
from the library's operators: projections by ``gs_linear``, heads into the cache
by ``gs_rope_append``, one-token attention by ``gs_decode_attention``, tokens by
``gs_sample``.  The prompt is run once; its pages are then shared by all
continuations (``PagePool.fork``), each of which copies only the page that it
goes on writing.

    python -m paper_2609_26638_gb300.best_of_n --n 8 --new 32
"""
from __future__ import annotations

import argparse
import dataclasses
from typing import Dict, List, Optional

import torch

from . import gs
from .cache import PAGE_TOKENS, PagePool

EPS = 1e-6


@dataclasses.dataclass(frozen=True)
class Shape:
    """d_model, d_ffn and the projections' widths are multiples of 128, the vocabulary too."""
    n_layers: int = 2
    d_model: int = 256
    n_heads: int = 8
    n_kv_heads: int = 2
    head_dim: int = 64
    d_ffn: int = 512
    vocab: int = 4096
    rotary_dim: int = 32
    rope_layout: int = gs.ROPE_INTERLEAVED
    rope_theta: float = 10000.0

    @property
    def qkv_dim(self) -> int:
        return (self.n_heads + 2 * self.n_kv_heads) * self.head_dim


def random_weights(shape: Shape, seed: int = 0, device: str = "cuda:0") -> Dict[str, object]:
    """fp16 matrices N(0, 0.02 .. 0.05), gains near 1."""
    g = torch.Generator(device="cpu").manual_seed(seed)

    def mat(rows, cols, std):
        return (std * torch.randn(rows, cols, generator=g)).half().to(device)

    def gain(n):
        return (1 + 0.1 * torch.randn(n, generator=g)).bfloat16().to(device)

    s = shape
    layers = [dict(norm1=gain(s.d_model), qkv=mat(s.qkv_dim, s.d_model, 0.05), q_gain=gain(s.head_dim),
                   k_gain=gain(s.head_dim), o=mat(s.d_model, s.n_heads * s.head_dim, 0.05),
                   norm2=gain(s.d_model), gate_up=mat(2 * s.d_ffn, s.d_model, 0.05),
                   down=mat(s.d_model, s.d_ffn, 0.05)) for _ in range(s.n_layers)]
    return dict(embed=mat(s.vocab, s.d_model, 1.0), layers=layers, norm=gain(s.d_model),
                lm_head=mat(s.vocab, s.d_model, 0.1))


def check_weights(shape: Shape, weights: Dict[str, object], device) -> None:
    """Refuses weights that are not what ``random_weights`` makes for this shape:
    the kernels read them through pointers."""
    s = shape
    q, f, d = s.n_heads * s.head_dim, s.d_ffn, s.d_model
    layer = dict(norm1=(d,), qkv=(s.qkv_dim, d), q_gain=(s.head_dim,), k_gain=(s.head_dim,), o=(d, q),
                 norm2=(d,), gate_up=(2 * f, d), down=(d, f))
    layers = weights.get("layers", ())
    if len(layers) != s.n_layers:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "weights of another number of layers")
    want = [(weights, dict(embed=(s.vocab, d), norm=(d,), lm_head=(s.vocab, d)))]
    for held, shapes in want + [(w, layer) for w in layers]:
        for name, size in shapes.items():
            t = held.get(name)
            if (not isinstance(t, torch.Tensor) or t.shape != size or not t.is_contiguous()
                    or t.dtype != (torch.float16 if len(size) == 2 else torch.bfloat16)
                    or t.device != device or t.data_ptr() % 16):
                raise gs.GsError(gs.GS_ERR_INVALID_ARG,
                                 f"{name}: contiguous, 16-byte aligned "
                                 f"{'fp16' if len(size) == 2 else 'bf16'} {list(size)} on {device} needed")


def check_tokens(tokens, vocab: int) -> None:
    """Refuses ids outside the vocabulary.  Ids on the device are not read here."""
    t = torch.as_tensor(tokens)
    if t.dim() != 1 or t.is_floating_point() or t.is_complex():
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "tokens must be a list of whole numbers")
    if not t.is_cuda and t.numel() and not (0 <= int(t.min()) and int(t.max()) < vocab):
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "token id outside the vocabulary")


def check_runs(runs, max_rows: int) -> int:
    """The tokens of all (sequence, first slot, tokens) runs; refuses runs that
    are empty, too many, or name a slot twice."""
    if not runs or any(len(t) == 0 for _, _, t in runs):
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "no tokens")
    rows = sum(len(t) for _, _, t in runs)
    if rows > max_rows:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "more tokens than max_rows")
    spans = sorted((s, first, first + len(t)) for s, first, t in runs)
    if any(a[0] == b[0] and b[1] < a[2] for a, b in zip(spans, spans[1:])):
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "two runs name one slot")
    return rows


class StepDecoder:
    """Feeds tokens of any sequences through the decoder, one call per step.
    The weights are used where they are (``random_weights`` shows their form).

    ``feed`` takes (sequence, first slot, tokens) runs: a prompt is one long run,
    a decode step one token per sequence.  Runs of one token go through
    ``gs_decode_attention`` together; in a longer run the tokens are rows over
    the same pages, each seeing the keys up to its own.  Runs of one call may
    follow one another in a sequence, but not name a slot twice.  A token id outside the
    vocabulary is refused; where the ids are on the device, it is clamped, and the
    next ``check`` raises.

    The work runs on a stream of the decoder's own (``stream``), ordered with the
    caller's current stream: tokens may come from work enqueued there, and what
    ``feed`` returns may be used there without synchronising."""

    def __init__(self, shape: Shape, weights: Dict[str, object], *, n_pages: int, max_seqs: int,
                 max_ctx: int, max_rows: int = 512, device: str = "cuda:0"):
        self.shape, self.w, self.max_rows = shape, weights, max_rows
        self.device = torch.empty(0, device=device).device            # (with its index)
        check_weights(shape, weights, self.device)
        self.stream = torch.cuda.Stream(self.device)
        torch.cuda.synchronize(self.device)
        self.pool = PagePool(n_layers=shape.n_layers, n_pages=n_pages, n_kv_heads=shape.n_kv_heads,
                             head_dim=shape.head_dim, dtype=torch.float16, max_seqs=max_seqs,
                             max_ctx=max_ctx, device=device, stream=self.stream)
        with torch.cuda.stream(self.stream):
            self.table = torch.empty(max_ctx, shape.rotary_dim // 2, 2, device=self.device)
            scaling = gs.gs_rope_scaling(kind=gs.ROPE_PLAIN, theta=shape.rope_theta)
            gs.gs_rope_table(scaling, shape.rotary_dim, max_ctx, self.table.data_ptr(),
                             self.stream.cuda_stream)
            need = max(gs.gs_decode_attention_scratch_bytes(self.pool.layer(0), r, shape.n_heads, 0)
                       for r in range(1, max_rows + 1))
            self.attn_scratch = torch.zeros(need, dtype=torch.uint8, device=self.device)
            wide = max(shape.qkv_dim, shape.d_model, 2 * shape.d_ffn, shape.vocab)
            need = max(gs.gs_linear_scratch_bytes(r, wide, 1) for r in range(1, max_rows + 1))
            # a scratch, and so an error word, for each product of a step: a call
            # clears its own
            self.gemm_scratch = torch.zeros(4 * shape.n_layers + 1, need, dtype=torch.uint8,
                                            device=self.device)
            self.gemm_err = torch.zeros((), dtype=torch.int32, device=self.device)
        self.rope = gs.gs_rope(self.table.data_ptr(), max_ctx, shape.rotary_dim, shape.rope_layout)

    def _linear(self, x, w, y, n_out: int, epilogue: int, at: int) -> None:
        """y = x w^T as the step's ``at``-th product."""
        scratch = self.gemm_scratch[at]
        gs.gs_linear(x.data_ptr(), w.data_ptr(), y.data_ptr(), x.shape[0], n_out, x.shape[1], epilogue,
                     1, scratch.data_ptr(), scratch.numel(), self.stream.cuda_stream)

    @staticmethod
    def _norm(h, gain):
        return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * gain.float()).half()

    def feed(self, runs) -> torch.Tensor:
        """fp16 logits [runs, vocab] after the last token of each run."""
        runs = list(runs)
        rows = check_runs(runs, self.max_rows)
        for _, _, t in runs:
            check_tokens(t, self.shape.vocab)
        caller = torch.cuda.current_stream(self.device)
        self.stream.wait_stream(caller)
        for _, _, t in runs:
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(self.stream)
        self.pool.prepare([(s, first, len(t)) for s, first, t in runs])
        with torch.cuda.stream(self.stream):
            logits = self._feed(runs, rows)
        caller.wait_stream(self.stream)
        logits.record_stream(caller)
        return logits

    def _feed(self, runs, rows):
        s, st = self.shape, self.stream.cuda_stream
        dev = self.device

        def ids(values):
            return torch.tensor(values, dtype=torch.int32).to(dev)
        seq = ids([q for q, _, t in runs for _ in t])
        slot = ids([first + i for _, first, t in runs for i in range(len(t))])
        n = slot + 1                       # a token sees itself and what lies before it
        token = torch.cat([torch.as_tensor(t, dtype=torch.int64, device=dev) for _, _, t in runs])
        inside = token.clamp(0, s.vocab - 1)
        self.pool.err.logical_or_((inside != token).any())
        h = self.w["embed"][inside].float()
        qkv = torch.empty(rows, s.qkv_dim, dtype=torch.float16, device=dev)
        out = torch.empty(rows, s.n_heads * s.head_dim, dtype=torch.float16, device=dev)
        act = torch.empty(rows, s.d_ffn, dtype=torch.float16, device=dev)
        width = s.n_heads * s.head_dim
        for i, w in enumerate(self.w["layers"]):
            cache = self.pool.layer(i)
            self._linear(self._norm(h, w["norm1"]), w["qkv"], qkv, s.qkv_dim, gs.EPI_STORE_F16, 4 * i)
            # queries in place: the key and value parts of qkv are read by the same call
            gs.gs_rope_append(cache, self.rope, qkv.data_ptr(), s.qkv_dim, rows, s.n_heads,
                              w["q_gain"].data_ptr(), w["k_gain"].data_ptr(), EPS, seq.data_ptr(),
                              slot.data_ptr(), slot.data_ptr(), qkv.data_ptr(), s.qkv_dim,
                              self.pool.err.data_ptr(), st)
            gs.gs_decode_attention(cache, qkv.data_ptr(), s.qkv_dim, seq.data_ptr(), n.data_ptr(), rows,
                                   s.n_heads, s.head_dim ** -0.5, 0, out.data_ptr(), width, 0, 0,
                                   self.attn_scratch.data_ptr(), self.attn_scratch.numel(), st)
            self._linear(out, w["o"], h, s.d_model, gs.EPI_RESID_F32, 4 * i + 1)
            self._linear(self._norm(h, w["norm2"]), w["gate_up"], act, s.d_ffn, gs.EPI_SWIGLU,
                         4 * i + 2)
            self._linear(act, w["down"], h, s.d_model, gs.EPI_RESID_F32, 4 * i + 3)
        last = torch.tensor([len(t) for _, _, t in runs]).cumsum(0).to(dev) - 1
        x = self._norm(h[last], self.w["norm"])
        logits = torch.empty(len(runs), s.vocab, dtype=torch.float16, device=dev)
        self._linear(x, self.w["lm_head"], logits, s.vocab, gs.EPI_STORE_F16, 4 * s.n_layers)
        words = self.gemm_scratch[:, :4].view(torch.int32)
        torch.maximum(self.gemm_err, words.amax(), out=self.gemm_err)
        return logits

    def check(self) -> None:
        """Synchronise and raise if a kernel met an index out of range, or a
        product a value beyond fp16's.  All error words are clear afterwards."""
        self.stream.synchronize()
        with torch.cuda.stream(self.stream):
            attn = self.attn_scratch[:4].view(torch.int32)
            attend, linear = int(attn.item()), int(self.gemm_err.item())
            attn.zero_()
            self.gemm_err.zero_()
        self.pool.check()
        if attend:
            raise gs.GsError(gs.GS_ERR_DEVICE_CHECK, "gs_decode_attention")
        if linear:
            raise gs.GsError(gs.GS_ERR_TIMEOUT if linear == 2 else gs.GS_ERR_DEVICE_CHECK, "gs_linear")


LOGIT_TYPES = {torch.float16: gs.GS_F16, torch.bfloat16: gs.GS_BF16, torch.float32: gs.GS_F32}


class Sampler:
    """gs_sample with one set of settings for every row."""

    def __init__(self, rows: int, *, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                 min_p: float = 0.0, device: str = "cuda:0"):
        def full(v, dtype=torch.float32):
            return torch.full((rows,), v, dtype=dtype, device=device)
        self._t = [full(temperature), full(top_p), full(min_p), full(top_k, torch.int32)]
        self._p = gs.gs_sample_params(*[t.data_ptr() for t in self._t])
        self.token = full(0, torch.int32)
        self.logprob = full(0.0)

    def draw(self, logits: torch.Tensor, u: torch.Tensor, stream) -> None:
        """token and logprob of each row, from uniforms ``u`` on ``stream``.

        logits: [rows, vocab] in 16 or 32 bits, neighbouring columns, no more rows
        than the sampler was made for; u: contiguous fp32 [rows]."""
        code = LOGIT_TYPES.get(logits.dtype)
        if (code is None or logits.dim() != 2 or logits.stride(1) != 1
                or logits.stride(0) < logits.shape[1] or logits.shape[0] > self.token.shape[0]
                or logits.device != self.token.device):
            raise gs.GsError(gs.GS_ERR_INVALID_ARG, "logits do not fit the sampler")
        if (u.dtype != torch.float32 or u.shape != logits.shape[:1] or not u.is_contiguous()
                or u.device != self.token.device):
            raise gs.GsError(gs.GS_ERR_INVALID_ARG, "uniforms do not fit the logits")
        with torch.cuda.stream(stream):
            gs.gs_sample(logits.data_ptr(), logits.stride(0), logits.shape[0], logits.shape[1], code,
                         self._p, u.data_ptr(), self.token.data_ptr(), self.logprob.data_ptr(), 0,
                         stream.cuda_stream)


def uniform_table(uniforms, new: int, n: int, device) -> torch.Tensor:
    """``uniforms`` as the kernel reads them: [new, n] contiguous fp32 on the device."""
    u = torch.as_tensor(uniforms)
    if u.shape != (new, n) or u.is_complex():
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "uniforms must be [new, n]")
    return u.to(device=device, dtype=torch.float32).contiguous()


def best_of_n(dec: StepDecoder, prompt: List[int], n: int, new: int, uniforms: Optional[torch.Tensor]
              = None, seed: int = 0, **settings):
    """n continuations of ``new`` tokens; (tokens [n, new], sum of log-probabilities [n]).

    uniforms: [new, n] numbers in [0, 1), or drawn from ``seed``.  The
    results are complete when the call returns (it synchronises)."""
    if not prompt or n < 1 or new < 0:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "an empty prompt, n < 1 or new < 0")
    if (new > 1 and n > dec.max_rows) or len(prompt) + max(new - 1, 0) > dec.pool.table.max_ctx:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "more sequences or tokens than the decoder was made for")
    caller = torch.cuda.current_stream(dec.device)
    dec.stream.wait_stream(caller)
    with torch.cuda.stream(dec.stream):
        if uniforms is None:
            g = torch.Generator(device=dec.device).manual_seed(seed)
            uniforms = torch.rand(new, n, device=dec.device, generator=g)
        else:
            uniforms = uniform_table(uniforms, new, n, dec.device)
            uniforms.record_stream(dec.stream)
        sampler = Sampler(n, device=str(dec.device), **settings)
        total = torch.zeros(n, device=dec.device)
        tokens = torch.empty(n, new, dtype=torch.int32, device=dec.device)
    seqs: List[int] = []
    try:
        seqs.append(dec.pool.open())
        for at in range(0, len(prompt), dec.max_rows):
            logits = dec.feed([(seqs[0], at, prompt[at: at + dec.max_rows])])
        seqs += dec.pool.fork(seqs[0], n - 1)
        with torch.cuda.stream(dec.stream):
            logits = logits.expand(n, -1).contiguous()
        for i in range(new):
            with torch.cuda.stream(dec.stream):
                sampler.draw(logits, uniforms[i], dec.stream)
                tokens[:, i] = sampler.token
                total += sampler.logprob
            if i + 1 < new:
                logits = dec.feed([(q, len(prompt) + i, sampler.token[j: j + 1])
                                   for j, q in enumerate(seqs)])
        dec.check()
    finally:
        for q in seqs:
            dec.pool.close(q)
    tokens.record_stream(caller)
    total.record_stream(caller)
    return tokens, total


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--n", type=int, default=8)
    ap.add_argument("--new", type=int, default=32)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-p", type=float, default=0.95)
    a = ap.parse_args()
    shape = Shape()
    ctx = a.prompt + a.new
    pages = (a.prompt // PAGE_TOKENS + 1) + a.n * (a.new // PAGE_TOKENS + 2)
    dec = StepDecoder(shape, random_weights(shape), n_pages=pages, max_seqs=a.n, max_ctx=ctx)
    prompt = torch.randint(0, shape.vocab, (a.prompt,), generator=torch.Generator().manual_seed(1)).tolist()
    tokens, logprob = best_of_n(dec, prompt, a.n, a.new, temperature=a.temperature, top_p=a.top_p)
    best = int(logprob.argmax())
    print(f"best of {a.n}: continuation {best}, log-probability {float(logprob[best]):.2f}")
    print(tokens[best].tolist())


if __name__ == "__main__":
    main()
