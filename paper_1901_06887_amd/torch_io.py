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
_DTYPES = {torch.float32: B.MT_F32, torch.bfloat16: B.MT_BF16}
_SCALES = (torch.float8_e8m0fnu, torch.uint8)


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError("%s of %s: float32 or bfloat16 is wanted" % (what, t.dtype))
    return code


def _rows(t: torch.Tensor, what: str, rows: int, width: int, dtypes, device: int) -> int:
    """The elements between consecutive rows of a [rows][width] tensor on the device, whose rows are contiguous."""
    if t.shape != (rows, width) or t.dtype not in dtypes or t.get_device() != device or (width > 1 and t.stride(1) != 1):
        raise ValueError("%s: %s %s %s with strides %s; [%d, %d] of %s with contiguous rows on cuda:%d is wanted"
                         % (what, tuple(t.shape), t.dtype, t.device, t.stride(), rows, width, " or ".join(str(d) for d in dtypes), device))
    return t.stride(0) if rows > 1 else max(t.stride(0), width)


def _list(t: torch.Tensor, what: str, n: int, dtype, device: int) -> None:
    if t.shape != (n,) or t.dtype != dtype or t.get_device() != device or (n > 1 and t.stride(0) != 1):
        raise ValueError("%s: %s %s %s; a contiguous [%d] of %s on cuda:%d is wanted" % (what, tuple(t.shape), t.dtype, t.device, n, dtype, device))


def _stream(stream: Optional[torch.cuda.Stream], device: int) -> int:
    # (the raw handle: a Stream object made per call takes as long as the rest of a small call)
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device)


def add_norm(ctx: B.Context, x: torch.Tensor, residual: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None,
             gain_ids: Optional[torch.Tensor] = None, eps: float = 1e-6, sum_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             out8: Optional[torch.Tensor] = None, out8_scales: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_add_norm on the given (or current) stream: h = x + residual into sum_out, h / rms(h) * gain into out (in x's type) and, as
    8-bit rows, into out8 (float8_e4m3fn) and out8_scales (float8_e8m0fnu).  gain: float32 [width], or [tenants, width] with
    gain_ids int32 [rows]."""
    code, (rows, width), dev = _dtype(x, "rows"), x.shape, x.get_device()
    same = (x.dtype,)
    a = B.mt_norm_args()
    a.rows, a.width, a.dtype, a.eps = rows, width, code, eps
    a.x, a.x_stride = x.data_ptr(), _rows(x, "x", rows, width, same, ctx.cfg.device)
    if residual is not None:
        a.residual, a.residual_stride = residual.data_ptr(), _rows(residual, "residual", rows, width, same, dev)
    if gain is not None:
        g = gain if gain.dim() == 2 else gain.unsqueeze(0)
        a.gain, a.gain_stride, a.n_gains = g.data_ptr(), _rows(g, "gain", g.shape[0], width, (torch.float32,), dev), g.shape[0]
    if gain_ids is not None:
        _list(gain_ids, "gain_ids", rows, torch.int32, dev)
        a.gain_ids = gain_ids.data_ptr()
    if sum_out is not None:
        a.sum, a.sum_stride = sum_out.data_ptr(), _rows(sum_out, "sum_out", rows, width, same, dev)
    if out is not None:
        a.y, a.y_stride = out.data_ptr(), _rows(out, "out", rows, width, same, dev)
    if out8 is not None:
        a.y8, a.y8_stride = out8.data_ptr(), _rows(out8, "out8", rows, width, (torch.float8_e4m3fn,), dev)
    if out8_scales is not None:
        a.y8_scales, a.y8_scales_stride = out8_scales.data_ptr(), _rows(out8_scales, "out8_scales", rows, -(-width // B.MT_MX_BLOCK), _SCALES, dev)
    ctx.add_norm(_stream(stream, dev), a)


def linear4(ctx: B.Context, groups, x: torch.Tensor, out: torch.Tensor, x_scales: Optional[torch.Tensor] = None, act: int = B.MT_ACT_NONE,
            stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_linear4 on the given (or current) stream: the rows of every group (row_groups) times its matrix, into out (float32 or bfloat16).
    x: float32, bfloat16, or float8_e4m3fn with x_scales."""
    rows, width = x.shape
    dev = ctx.cfg.device
    a = B.mt_linear4_args()
    if x.dtype == torch.float8_e4m3fn:
        a.x_dtype = B.MT_MX8
        if x_scales is None:
            raise ValueError("8-bit rows come with their scales")
        a.x_scales, a.x_scales_stride = x_scales.data_ptr(), _rows(x_scales, "x_scales", rows, -(-width // B.MT_MX_BLOCK), _SCALES, dev)
    else:
        a.x_dtype = _dtype(x, "rows")
        if x_scales is not None:
            raise ValueError("scales come with 8-bit rows only")
    a.rows, a.act, a.y_dtype = rows, act, _dtype(out, "out")
    a.x, a.y = x.data_ptr(), out.data_ptr()
    # (a matrix may be narrower than the rows, so the widths that the strides are checked against are these)
    a.x_stride, a.y_stride = _rows(x, "x", rows, width, (x.dtype,), dev), _rows(out, "out", rows, out.shape[1], (out.dtype,), dev)
    if rows <= 1:
        a.x_stride, a.y_stride = width, out.shape[1]
    ctx.linear4(_stream(stream, dev), a, groups)


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
    code, (rows, classes), dev = _dtype(logits, "logits"), logits.shape, ctx.cfg.device
    a = B.mt_score_args()
    a.rows, a.classes, a.dtype, a.temperature = rows, classes, code, temperature
    a.logits, a.row_stride = logits.data_ptr(), _rows(logits, "logits", rows, classes, (logits.dtype,), dev)
    _list(out.entropy, "entropy", rows, torch.float32, dev)
    a.entropy = out.entropy.data_ptr()
    if n_classes is not None:
        _list(n_classes, "n_classes", rows, torch.int32, dev)
        a.n_classes = n_classes.data_ptr()
    if allowed is not None:
        if allowed.dim() != 2 or allowed.shape[1] < -(-classes // 32):
            raise ValueError("allowed: %s for %d rows of %d classes" % (tuple(allowed.shape), rows, classes))
        a.allowed, a.allowed_stride = allowed.data_ptr(), _rows(allowed, "allowed", rows, allowed.shape[1], (torch.int32,), dev)
    if (given is None) != (out.given_ranks is None):
        raise ValueError("given classes and their outputs come together")
    if given is not None:
        n = out.given_ranks.shape[1]
        for t, what, d in ((given, "given", torch.int32), (out.given_ranks, "given_ranks", torch.int32), (out.given_logprobs, "given_logprobs", torch.float32)):
            if _rows(t, what, rows, n, (d,), dev) != n:
                raise ValueError("%s is not contiguous" % what)
        a.n_given, a.given, a.given_ranks, a.given_logprobs = n, given.data_ptr(), out.given_ranks.data_ptr(), out.given_logprobs.data_ptr()
    if out.top_ids is not None:
        n = out.top_ids.shape[1]
        for t, what, d in ((out.top_ids, "top_ids", torch.int32), (out.top_logprobs, "top_logprobs", torch.float32)):
            if _rows(t, what, rows, n, (d,), dev) != n:
                raise ValueError("%s is not contiguous" % what)
        a.top, a.top_ids, a.top_logprobs = n, out.top_ids.data_ptr(), out.top_logprobs.data_ptr()
    a.scratch, a.scratch_bytes = out.scratch.data_ptr(), out.scratch.numel()
    ctx.score(_stream(stream, dev), a)
    return out
