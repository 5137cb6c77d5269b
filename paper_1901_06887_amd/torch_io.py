"""Glue between torch device tensors and the C ABI: allocation of the caller-owned buffers
and pointer passing.  No arithmetic happens here."""
from __future__ import annotations

from dataclasses import dataclass
from typing import Dict, Optional

import numpy as np
import torch

from . import binding as B


@dataclass
class Served:
    labels: torch.Tensor      # int32 [R]
    probs: torch.Tensor       # float32 [R, row_stride]
    logits: torch.Tensor      # float32 [R, row_stride]
    n_classes: torch.Tensor   # int32 [R]


def specs_of(layers) -> list:
    """mt_layer_spec list from objects with kind/act/in_features/out_features/in_h/in_w/stride (and, where they
    have them, ksize/pad/src/src2)."""
    return [B.layer_spec(l.kind, l.act, l.in_features, l.out_features, l.in_h, l.in_w, l.stride,
                         getattr(l, "ksize", 3), getattr(l, "pad", 1), getattr(l, "src", 0), getattr(l, "src2", 0)) for l in layers]


def context_for(tenants: Dict[int, object], dtype: str, max_requests: int, device: int = 0,
                max_tenants: Optional[int] = None, arena_slack: float = 1.05, run_slots: int = 1,
                arena_bytes: Optional[int] = None, cache: bool = False) -> B.Context:
    """A context sized for the given tenant models (objects with .layers/.weights/.biases); the
    sizes come from the library's own account of every model (mt_model_footprint_get)."""
    code = B.MT_F32 if dtype == "f32" else B.MT_BF16
    width, classes, arena = 64, 1, 0
    for m in tenants.values():
        f = B.model_footprint(specs_of(m.layers), code)
        width, classes, arena = max(width, f["min_width"]), max(classes, f["n_classes"]), arena + f["arena_bytes"]
    T = max_tenants if max_tenants is not None else (max(tenants) + 1 if tenants else 1)
    return B.Context(T, max_requests, width, classes, arena_bytes if arena_bytes is not None else int(arena * arena_slack) + (1 << 20),
                     code, device, run_slots, cache)


def register_tenants(ctx: B.Context, tenants: Dict[int, object]):
    for t, m in tenants.items():
        ctx.register_model(int(t), specs_of(m.layers), m.weights, m.biases, getattr(m, "bn", None), getattr(m, "bn_eps", 1e-5))


def to_device(x: np.ndarray, dtype: str, device="cuda:0") -> torch.Tensor:
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    if dtype == "bf16":
        t = t.to(torch.bfloat16)
    return t.to(device)


def alloc_outputs(n: int, row_stride: int, device="cuda:0") -> Served:
    return Served(torch.empty(n, dtype=torch.int32, device=device),
                  torch.empty((n, row_stride), dtype=torch.float32, device=device),
                  torch.empty((n, row_stride), dtype=torch.float32, device=device),
                  torch.empty(n, dtype=torch.int32, device=device))


def serve(ctx: B.Context, tenant_ids: torch.Tensor, inputs: torch.Tensor, out: Optional[Served] = None,
          stream: Optional[torch.cuda.Stream] = None, static: bool = False) -> Served:
    """mt_submit_batch + mt_run (mt_run_static with `static`) on the given (or current) stream; returns
    without synchronising."""
    n = int(tenant_ids.numel())
    assert tenant_ids.dtype == torch.int32 and tenant_ids.is_cuda and inputs.is_cuda and inputs.is_contiguous()
    if out is None:
        out = alloc_outputs(n, ctx.cfg.max_classes, inputs.device)
    s = stream if stream is not None else torch.cuda.current_stream(inputs.device)
    ctx.submit_batch(tenant_ids.data_ptr(), inputs.data_ptr(), n, inputs.shape[1])
    (ctx.run_static if static else ctx.run)(s.cuda_stream, out.labels.data_ptr(), out.probs.data_ptr(), out.logits.data_ptr(),
            out.n_classes.data_ptr(), out.labels.numel(), out.probs.shape[1])
    return out


# ---- operators behind language models' answers ---------------------------------------------------
# (A small call takes the GPU 3 to 5 us and the library's launch 3 us of the host, so the checks here look every attribute up once and the argument
# blocks are packed in one go.)
_F32, _BF16, _I32, _E4M3, _E8M0 = torch.float32, torch.bfloat16, torch.int32, torch.float8_e4m3fn, torch.float8_e8m0fnu
_DTYPES = {_F32: B.MT_F32, _BF16: B.MT_BF16}
_raw_stream = torch._C._cuda_getCurrentRawStream


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError("%s of %s: float32 or bfloat16 is wanted" % (what, t.dtype))
    return code


def _rows(t: torch.Tensor, what: str, rows: int, width: int, dtype, device: int, or_dtype=None) -> int:
    """The elements between consecutive rows of a [rows][width] tensor on the device, whose rows are contiguous."""
    shape, strides, d = t.shape, t.stride(), t.dtype
    if len(shape) != 2 or shape[0] != rows or shape[1] != width or (d is not dtype and d is not or_dtype) or t.get_device() != device or (strides[1] != 1 and width > 1):
        raise ValueError("%s: %s %s %s with strides %s; [%d, %d] of %s with contiguous rows on cuda:%d is wanted"
                         % (what, tuple(shape), d, t.device, strides, rows, width, dtype, device))
    return strides[0] if rows > 1 else width


def _list(t: torch.Tensor, what: str, n: int, dtype, device: int) -> int:
    """The address of a contiguous list on the device."""
    if t.shape != (n,) or t.dtype is not dtype or t.get_device() != device or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s: %s %s %s; a contiguous [%d] of %s on cuda:%d is wanted" % (what, tuple(t.shape), t.dtype, t.device, n, dtype, device))
    return t.data_ptr()


def _table(t: torch.Tensor, what: str, rows: int, width: int, dtype, device: int) -> int:
    """The address of a contiguous [rows][width] tensor on the device."""
    if _rows(t, what, rows, width, dtype, device) != width:
        raise ValueError("%s is not contiguous" % what)
    return t.data_ptr()


def _matrix(t: torch.Tensor, what: str):
    if t.dim() != 2:
        raise ValueError("%s: %s; two dimensions are wanted" % (what, tuple(t.shape)))
    return t.shape


def add_norm(ctx: B.Context, x: torch.Tensor, residual: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None,
             gain_ids: Optional[torch.Tensor] = None, eps: float = 1e-6, sum_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             out8: Optional[torch.Tensor] = None, out8_scales: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_add_norm on the given (or current) stream: h = x + residual into sum_out, h / rms(h) * gain into out (in x's type) and, as
    8-bit rows, into out8 (float8_e4m3fn) and out8_scales (float8_e8m0fnu, or its bytes).  gain: float32 [width], or [tenants, width] with
    gain_ids int32 [rows]."""
    (rows, width), dev, dtype = _matrix(x, "x"), ctx.device, x.dtype
    code = _dtype(x, "rows")
    x_stride = _rows(x, "x", rows, width, dtype, dev)
    residual_p = residual_stride = gain_p = gain_stride = n_gains = ids_p = sum_p = sum_stride = y_p = y_stride = y8_p = y8_stride = scales_p = scales_stride = 0
    if residual is not None:
        residual_p, residual_stride = residual.data_ptr(), _rows(residual, "residual", rows, width, dtype, dev)
    if gain is not None:
        if gain.dim() == 1:
            gain = gain.unsqueeze(0)
        n_gains = gain.shape[0]
        gain_p, gain_stride = gain.data_ptr(), _rows(gain, "gain", n_gains, width, _F32, dev)
    if gain_ids is not None:
        ids_p = _list(gain_ids, "gain_ids", rows, _I32, dev)
    if sum_out is not None:
        sum_p, sum_stride = sum_out.data_ptr(), _rows(sum_out, "sum_out", rows, width, dtype, dev)
    if out is not None:
        y_p, y_stride = out.data_ptr(), _rows(out, "out", rows, width, dtype, dev)
    if out8 is not None:
        y8_p, y8_stride = out8.data_ptr(), _rows(out8, "out8", rows, width, _E4M3, dev)
    if out8_scales is not None:
        scales_p, scales_stride = out8_scales.data_ptr(), _rows(out8_scales, "out8_scales", rows, (width + 31) // 32, _E8M0, dev, torch.uint8)
    ctx.add_norm(stream.cuda_stream if stream is not None else _raw_stream(dev),
                 B.pack_norm_args(x.data_ptr(), residual_p, gain_p, ids_p, sum_p, y_p, y8_p, scales_p, x_stride, residual_stride, gain_stride, sum_stride, y_stride,
                                  y8_stride, scales_stride, rows, width, n_gains, code, eps, 0))


def linear4(ctx: B.Context, groups, x: torch.Tensor, out: torch.Tensor, x_scales: Optional[torch.Tensor] = None, act: int = B.MT_ACT_NONE,
            stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_linear4 on the given (or current) stream: the rows of every group (row_groups) times its matrix, into out (float32 or bfloat16).
    x: float32, bfloat16, or float8_e4m3fn with x_scales."""
    (rows, width), dev, dtype = _matrix(x, "x"), ctx.device, x.dtype
    scales_p = scales_stride = 0
    if dtype is _E4M3:
        code = B.MT_MX8
        if x_scales is None:
            raise ValueError("8-bit rows come with their scales")
        scales_p, scales_stride = x_scales.data_ptr(), _rows(x_scales, "x_scales", rows, (width + 31) // 32, _E8M0, dev, torch.uint8)
    else:
        code = _dtype(x, "rows")
        if x_scales is not None:
            raise ValueError("scales come with 8-bit rows only")
    n = _matrix(out, "out")[1]
    # (a matrix may be narrower than the rows: its sizes are checked against the strides, which for one row are the widths)
    ctx.linear4(stream.cuda_stream if stream is not None else _raw_stream(dev),
                B.pack_linear4_args(x.data_ptr(), scales_p, out.data_ptr(), _rows(x, "x", rows, width, dtype, dev), scales_stride,
                                    _rows(out, "out", rows, n, out.dtype, dev), rows, code, _dtype(out, "out"), act), groups)


@dataclass
class Scores:
    given_logprobs: Optional[torch.Tensor]   # float32 [R, n_given]
    given_ranks: Optional[torch.Tensor]      # int32 [R, n_given]
    entropy: torch.Tensor                    # float32 [R]
    top_ids: Optional[torch.Tensor]          # int32 [R, top]
    top_logprobs: Optional[torch.Tensor]     # float32 [R, top]
    scratch: torch.Tensor                    # uint8: what the workgroups that share a row hand over


def alloc_scores(rows: int, n_given: int = 0, top: int = 0, device="cuda:0", classes: int = 0) -> Scores:
    """Outputs and scratch of mt_score for so many rows (of so many classes; 0: of any number).  One call at a time may use them."""
    pair = lambda n: (torch.empty((rows, n), dtype=torch.float32, device=device), torch.empty((rows, n), dtype=torch.int32, device=device)) if n else (None, None)  # noqa: E731
    (lp, ranks), (top_lp, ids) = pair(n_given), pair(top)
    scratch = torch.zeros(B.score_scratch(rows, classes or 0x7fffffff, n_given, top), dtype=torch.uint8, device=device)
    return Scores(lp, ranks, torch.empty(rows, dtype=torch.float32, device=device), ids, top_lp, scratch)


def score(ctx: B.Context, logits: torch.Tensor, out: Scores, given: Optional[torch.Tensor] = None, n_classes: Optional[torch.Tensor] = None,
          allowed: Optional[torch.Tensor] = None, temperature: float = 1.0, stream: Optional[torch.cuda.Stream] = None) -> Scores:
    """mt_score on the given (or current) stream: what rows of logits say about given classes (int32 [rows, n_given]), their entropy and
    the best alternatives.  n_classes: int32 [rows]; allowed: int32 [rows, words], a bit for every class."""
    (rows, classes), dev = _matrix(logits, "logits"), ctx.device
    code = _dtype(logits, "logits")
    stride = _rows(logits, "logits", rows, classes, logits.dtype, dev)
    n_p = allowed_p = allowed_stride = given_p = n_given = lp_p = ranks_p = top = ids_p = top_p = 0
    entropy_p = _list(out.entropy, "entropy", rows, _F32, dev)
    if n_classes is not None:
        n_p = _list(n_classes, "n_classes", rows, _I32, dev)
    if allowed is not None:
        words = _matrix(allowed, "allowed")[1]
        if words < (classes + 31) // 32:
            raise ValueError("allowed: %s for %d rows of %d classes" % (tuple(allowed.shape), rows, classes))
        allowed_p, allowed_stride = allowed.data_ptr(), _rows(allowed, "allowed", rows, words, _I32, dev)
    ranks = out.given_ranks
    if (given is None) != (ranks is None):
        raise ValueError("given classes and their outputs come together")
    if given is not None:
        n_given = ranks.shape[1]
        given_p, ranks_p = _table(given, "given", rows, n_given, _I32, dev), _table(ranks, "given_ranks", rows, n_given, _I32, dev)
        lp_p = _table(out.given_logprobs, "given_logprobs", rows, n_given, _F32, dev)
    if out.top_ids is not None:
        top = out.top_ids.shape[1]
        ids_p, top_p = _table(out.top_ids, "top_ids", rows, top, _I32, dev), _table(out.top_logprobs, "top_logprobs", rows, top, _F32, dev)
    scratch = out.scratch
    ctx.score(stream.cuda_stream if stream is not None else _raw_stream(dev),
              B.pack_score_args(logits.data_ptr(), n_p, allowed_p, given_p, lp_p, ranks_p, entropy_p, ids_p, top_p, scratch.data_ptr(), scratch.numel(), stride,
                                allowed_stride, rows, classes, n_given, top, code, temperature))
    return out
