"""4-bit weights for ``gs_qlinear``: quantized, packed and held.

A matrix [N, K] becomes whole numbers 0 .. 15 with a scale (and a zero) for each
``group`` of a row's neighbouring weights, (q - z) * s, laid out once in the order in
which the kernel reads it.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import gs

TYPES = {torch.float16: gs.GS_F16, torch.bfloat16: gs.GS_BF16}


def quantize(w: torch.Tensor, group: int = 64, zeros: bool = False
             ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """(q, scale, zero) of a 16-bit matrix: uint8 [N, K / 2] with the first of two
    weights in the low bits, scales of the matrix's type and zeros [N, K / group].

    Without zeros a group is spread evenly around 0 (z = 8), its largest magnitude at -8
    or 7; with them its least weight is 0 or below it, its largest 15."""
    if w.dim() != 2 or w.dtype not in TYPES or group not in (32, 64, 128) or w.shape[1] % group:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "a 16-bit [N, K] matrix with K a multiple of the group needed")
    if not torch.isfinite(w).all():
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "an infinite or NaN weight")
    x = w.contiguous().float().view(w.shape[0], -1, group)
    lo, hi = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
    exact = (hi - lo) / 15 if zeros else torch.maximum(-lo / 8, hi / 7)
    exact = torch.where(torch.isinf(exact), hi / 15 - lo / 15, exact)
    scale = exact.to(w.dtype)
    # below the type's normal numbers a rounding down could leave the largest weights out of reach
    short = scale.float() < exact * (1 - torch.finfo(w.dtype).eps)
    scale = torch.where(short, (scale.view(torch.int16) + 1).view(w.dtype), scale)
    step = torch.where(scale == 0, 1, scale.float())
    zero = (-lo / step).round().clamp(0, 15) if zeros else torch.full_like(step, 8.0)
    q = (x / step[..., None] + zero[..., None]).round().clamp(0, 15).to(torch.uint8).flatten(1)
    return q[:, 0::2] | (q[:, 1::2] << 4), scale, zero.to(torch.uint8) if zeros else None


class QWeight:
    """A packed matrix: ``desc`` is what ``gs_qlinear`` takes, valid as long as this lives.

    ``gated``: the rows are a SwiGLU's gate and, behind them, its up projection.  The
    packing runs on the current stream."""

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, zero: Optional[torch.Tensor] = None, *,
                 group: int, gated: bool = False):
        n, k = (q.shape[0], 2 * q.shape[1]) if q.dim() == 2 else (0, 0)
        want = (n, k // group if group > 0 else 0)
        held = [t for t in (q, scale, zero) if t is not None]
        if (q.dim() != 2 or q.dtype != torch.uint8 or scale.dtype not in TYPES or scale.shape != want
                or (zero is not None and (zero.dtype != torch.uint8 or zero.shape != want))
                or not all(t.is_cuda and t.device == q.device and t.is_contiguous() for t in held)):
            raise gs.GsError(gs.GS_ERR_INVALID_ARG, "q, scale and zero do not fit together")
        self.dtype, self.device = scale.dtype, q.device
        self.desc = gs.gs_qweight(0, n, k, group, TYPES[scale.dtype], int(zero is not None), int(gated))
        need = gs.gs_qweight_bytes(self.desc)
        if need == 0:
            raise gs.GsError(gs.GS_ERR_INVALID_ARG, "no such 4-bit matrix")
        with torch.cuda.device(q.device):
            self.packed = torch.empty(need, dtype=torch.uint8, device=q.device)
            self.desc.packed = self.packed.data_ptr()
            stream = torch.cuda.current_stream()
            gs.gs_qweight_pack(self.desc, q.data_ptr(), scale.data_ptr(),
                               zero.data_ptr() if zero is not None else 0, stream.cuda_stream)
        for t in held:
            t.record_stream(stream)

    @property
    def shape(self) -> Tuple[int, int]:
        return self.desc.N, self.desc.K

    @property
    def gated(self) -> bool:
        return bool(self.desc.gated)


def quantize_decoder(weights: Dict[str, object], group: int = 64, zeros: bool = False) -> Dict[str, object]:
    """A decoder's weights (``best_of_n.random_weights``) with every matrix but the
    embedding in 4 bits."""
    def of(w, gated=False):
        return QWeight(*quantize(w, group, zeros), group=group, gated=gated)
    layers = [{**w, **{k: of(w[k], k == "gate_up") for k in ("qkv", "o", "gate_up", "down")}}
              for w in weights["layers"]]
    return {**weights, "layers": layers, "lm_head": of(weights["lm_head"])}
