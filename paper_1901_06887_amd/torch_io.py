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
_raw_stream = torch._C._cuda_getCurrentRawStream
_answers = None


def answers():
    """The module of the calls on tensors (csrc/lm_torch.cpp), bound to the library; raises if it has not been built (no fallback path exists)."""
    global _answers
    if _answers is None:
        import ctypes
        lib = B.load_library()
        try:
            from . import _answers as calls
        except ImportError as e:
            raise ImportError("_answers.so is missing or was built for another torch: build it with `python -m paper_1901_06887_amd.build` (%s)" % e)
        calls.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (lib.mt_add_norm, lib.mt_linear4_within, lib.mt_score)))
        _answers = calls
    return _answers


def add_norm(ctx: B.Context, x: torch.Tensor, residual: Optional[torch.Tensor] = None, gain: Optional[torch.Tensor] = None,
             gain_ids: Optional[torch.Tensor] = None, eps: float = 1e-6, sum_out: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
             out8: Optional[torch.Tensor] = None, out8_scales: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_add_norm on the given (or current) stream: h = x + residual into sum_out, h / rms(h) * gain into out (in x's type) and, as
    8-bit rows, into out8 (float8_e4m3fn) and out8_scales (float8_e8m0fnu, or its bytes).  gain: float32 [width], or [tenants, width] with
    gain_ids int32 [rows].  Forward only, like the other operators: inputs may require gradients, no output carries one."""
    st = (_answers or answers()).add_norm(ctx._h.value or 0, stream.cuda_stream if stream is not None else _raw_stream(ctx.device), ctx.device, x, residual, gain, gain_ids,
                                          eps, sum_out, out, out8, out8_scales)
    if st:
        ctx._check(st)


def linear4(ctx: B.Context, groups, x: torch.Tensor, out: torch.Tensor, x_scales: Optional[torch.Tensor] = None, act: int = B.MT_ACT_NONE,
            stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_linear4 on the given (or current) stream: the rows of every group (row_groups) times its matrix, into out (float32 or bfloat16).
    x: float32, bfloat16, or float8_e4m3fn with x_scales.  Forward only."""
    st = (_answers or answers()).linear4(ctx._h.value or 0, stream.cuda_stream if stream is not None else _raw_stream(ctx.device), ctx.device, groups, x, out, x_scales, act)
    if st:
        ctx._check(st)


@dataclass
class Scores:
    """Outputs of mt_score; one that is set to None is left out."""
    given_logprobs: Optional[torch.Tensor]   # float32 [R, n_given]
    given_ranks: Optional[torch.Tensor]      # int32 [R, n_given]
    entropy: Optional[torch.Tensor]          # float32 [R]
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
    the best alternatives.  n_classes: int32 [rows]; allowed: int32 [rows, words], a bit for every class.  Forward only."""
    st = (_answers or answers()).score(ctx._h.value or 0, stream.cuda_stream if stream is not None else _raw_stream(ctx.device), ctx.device, logits, given, n_classes, allowed,
                                       temperature, out.given_logprobs, out.given_ranks, out.entropy, out.top_ids, out.top_logprobs, out.scratch)
    if st:
        ctx._check(st)
    return out
