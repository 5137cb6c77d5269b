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
        calls.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in (lib.mt_add_norm, lib.mt_linear4_within, lib.mt_score, lib.mt_kv_write, lib.mt_attend, lib.mt_kv_grow, lib.mt_kv_fork,
                                                                           lib.mt_kv_free, lib.mt_kv_compact, lib.mt_kv_copy, lib.mt_sample)))
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


# ---- caches of language models -----------------------------------------------------------------------
_KV_TYPES = {B.MT_F32: torch.float32, B.MT_BF16: torch.bfloat16, B.MT_KV8: torch.float8_e4m3fn}


class KVCache:
    """A paged cache (mt_kv_cache): its tensors, and their description as the calls take it.

    k [layers, pages, heads, page_tokens, head_dim], v [layers, pages, heads, head_dim, page_tokens]; with MT_KV8 k_scales, v_scales float8_e8m0fnu
    [layers, pages, heads, page_tokens]; table int32 [seqs, width], lengths int32 [seqs], refs int32 [pages], work uint8."""

    def __init__(self, k, v, k_scales, v_scales, table, lengths, refs, work, dtype: int):
        """A cache of the caller's own tensors, pages and layers as far apart as they like; refs and work may be None where no call on pages is made.  What does not fit is a ValueError."""
        want = _wanted
        kind = _KV_TYPES.get(dtype)
        want(kind is not None, "of dtype MT_F32, MT_BF16 or MT_KV8")
        kinds = (kind, torch.uint8) if dtype == B.MT_KV8 else (kind,)          # (8-bit values also as their bytes, scales too)
        want(isinstance(k, torch.Tensor) and k.dim() == 5 and k.dtype in kinds, "k %s [layers, pages, heads, page_tokens, head_dim]" % kind)
        layers, pages, heads, page_tokens, head_dim = k.shape
        page_stride, layer_stride = _blocks(k, "k", k.shape, kinds, k.device)
        want(_blocks(v, "v", (layers, pages, heads, head_dim, page_tokens), kinds, k.device) == (page_stride, layer_stride), "v of k's strides between pages and layers")
        scales = [(0, 0), (0, 0)]
        if dtype == B.MT_KV8:
            scales = [_blocks(t, name, (layers, pages, heads, page_tokens), (torch.float8_e8m0fnu, torch.uint8), k.device) for t, name in ((k_scales, "k_scales"), (v_scales, "v_scales"))]
        else:
            want(k_scales is None and v_scales is None, "scales with MT_KV8 only")
        want(scales[0] == scales[1], "v_scales of k_scales' strides")
        want(_fits(table, 2, torch.int32, k.device) and (table.shape[1] <= 1 or table.stride(1) == 1) and (table.shape[0] <= 1 or table.stride(0) >= table.shape[1]), "table int32 [seqs, width], rows side by side")
        want(_fits(lengths, 1, torch.int32, k.device) and lengths.numel() == table.shape[0] and lengths.is_contiguous(), "lengths int32 [%d], contiguous" % table.shape[0])
        want(refs is None or _fits(refs, 1, torch.int32, k.device) and refs.numel() == pages and refs.is_contiguous(), "refs int32 [%d], contiguous" % pages)
        want(work is None or _fits(work, 1, torch.uint8, k.device) and work.is_contiguous(), "work uint8, contiguous")
        self.k, self.v, self.k_scales, self.v_scales, self.table, self.lengths, self.refs, self.work = k, v, k_scales, v_scales, table, lengths, refs, work
        p = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.spec = B.mt_kv_cache(p(k), p(v), p(k_scales), p(v_scales), p(table), p(lengths), p(refs), p(work), page_stride, layer_stride, *scales[0],
                                  max(table.stride(0), table.shape[1]), 0 if work is None else work.numel(), dtype, layers, pages, heads, page_tokens, head_dim, table.shape[0], table.shape[1])
        self._tensors = (k, v, k_scales, v_scales, table, lengths, refs)      # (the spec has their addresses)


def _wanted(fits: bool, what: str) -> None:
    if not fits:
        raise ValueError("cache: %s wanted" % what)


def _fits(t, dims: int, dtype, device) -> bool:
    return isinstance(t, torch.Tensor) and t.dim() == dims and t.dtype == dtype and t.device == device


def _blocks(t, name: str, shape, dtypes, device):
    """Strides between pages and between layers of [layers, pages, ..], each page's block contiguous.  Where there is one alone: as if side by side."""
    _wanted(isinstance(t, torch.Tensor) and t.shape == torch.Size(shape) and t.dtype in dtypes and t.device == device, "%s %s %s on %s" % (name, dtypes[0], list(shape), device))
    block = 1
    for size, stride in zip(reversed(t.shape[2:]), reversed(t.stride()[2:])):
        _wanted(size <= 1 or stride == block, "%s with every page's elements side by side" % name)
        block *= size
    page = t.stride(1) if t.shape[1] > 1 else block
    return page, t.stride(0) if t.shape[0] > 1 else page * t.shape[1]


def alloc_kv(pages: int, page_tokens: int, heads: int, head_dim: int, seqs: int, width: int, dtype: int = B.MT_BF16, layers: int = 1, device="cuda:0") -> KVCache:
    """An empty cache of so many pages, for `seqs` sequences of up to `width` pages each.  dtype: MT_F32, MT_BF16 or MT_KV8."""
    if dtype not in _KV_TYPES:
        raise ValueError("a cache of dtype %r" % (dtype,))
    buf = lambda t, *shape: torch.empty(shape, dtype=t, device=device)  # noqa: E731
    scales = (lambda: buf(torch.uint8, layers, pages, heads, page_tokens).fill_(127).view(torch.float8_e8m0fnu)) if dtype == B.MT_KV8 else lambda: None
    return KVCache(buf(_KV_TYPES[dtype], layers, pages, heads, page_tokens, head_dim), buf(_KV_TYPES[dtype], layers, pages, heads, head_dim, page_tokens), scales(), scales(),
                   buf(torch.int32, seqs, width).fill_(-1), buf(torch.int32, seqs).zero_(), buf(torch.int32, pages).zero_(), buf(torch.uint8, B.kv_work(pages, seqs)), dtype)


def _where(ctx: B.Context, stream):
    return ctx._h.value or 0, stream.cuda_stream if stream is not None else _raw_stream(ctx.device), ctx.device


def kv_write(ctx: B.Context, cache: KVCache, k: torch.Tensor, v: torch.Tensor, seqs: Optional[torch.Tensor] = None, first_row: Optional[torch.Tensor] = None, max_new: int = 1,
             layer: int = 0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_write on the given (or current) stream: keys and values [rows, heads * head_dim] of the last tokens of every sequence into their pages.  seqs: int32, the
    sequences of the batch (None: 0, 1, ...); first_row: int32, one more than there are (None: a row each); max_new: most rows of a sequence."""
    st = (_answers or answers()).kv_write(*_where(ctx, stream), cache.spec, cache._tensors, k, v, seqs, first_row, max_new, layer)
    if st:
        ctx._check(st)


def alloc_attend(ctx: B.Context, cache: KVCache, q_heads: int, n_seqs: int, max_new: int = 1, max_length: int = 0) -> torch.Tensor:
    """Scratch of mt_attend for batches of so many sequences.  One call at a time may use it."""
    return torch.zeros(B.attend_scratch(cache.spec, n_seqs, q_heads, max_new, max_length), dtype=torch.uint8, device=cache.k.device)


def attend(ctx: B.Context, cache: KVCache, q: torch.Tensor, out: torch.Tensor, seqs: Optional[torch.Tensor] = None, first_row: Optional[torch.Tensor] = None, max_new: int = 1,
           max_length: int = 0, window: int = 0, scale: Optional[float] = None, lse: Optional[torch.Tensor] = None, layer: int = 0, scratch: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_attend on the given (or current) stream: rows q [rows, q_heads * head_dim] of the last tokens of every sequence (whose keys and values are written already)
    attend to all of it, each up to itself; out like q, lse float32 [rows, q_heads].  seqs, first_row, max_new: as in kv_write.  max_length: tokens of the longest sequence
    (0: what the table holds).  window: tokens that a row sees (0: all).  scale: None for head_dim^-0.5.  scratch: alloc_attend's for the same sizes.  Forward only."""
    st = (_answers or answers()).attend(*_where(ctx, stream), cache.spec, cache._tensors, q, out, seqs, first_row, max_new, layer, window, max_length, scale, lse, scratch)
    if st:
        ctx._check(st)


def kv_grow(ctx: B.Context, cache: KVCache, tokens: torch.Tensor, seqs: Optional[torch.Tensor] = None, granted: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_grow: room for tokens[i] (int32) more tokens of sequence seqs[i] (None: i); granted[i] says whether there was."""
    st = (_answers or answers()).kv_grow(*_where(ctx, stream), cache.spec, cache._tensors, seqs, tokens, granted)
    if st:
        ctx._check(st)


def kv_fork(ctx: B.Context, cache: KVCache, parents: torch.Tensor, children: torch.Tensor, granted: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_fork: the empty sequence children[i] becomes a copy of parents[i] that shares its full pages."""
    st = (_answers or answers()).kv_fork(*_where(ctx, stream), cache.spec, cache._tensors, parents, children, granted)
    if st:
        ctx._check(st)


def kv_free(ctx: B.Context, cache: KVCache, seqs: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_free: the sequences let go of their pages."""
    st = (_answers or answers()).kv_free(*_where(ctx, stream), cache.spec, cache._tensors, seqs)
    if st:
        ctx._check(st)


def kv_compact(ctx: B.Context, cache: KVCache, live: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_compact: held pages move to the lowest numbers; live (int32 [1]) receives how many there are."""
    st = (_answers or answers()).kv_compact(*_where(ctx, stream), cache.spec, cache._tensors, live)
    if st:
        ctx._check(st)


def kv_copy(ctx: B.Context, cache: KVCache, from_pages: torch.Tensor, to_pages: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """mt_kv_copy: pages of all layers copied over others, none of them another pair's target (a chain takes a call for each link)."""
    st = (_answers or answers()).kv_copy(*_where(ctx, stream), cache.spec, cache._tensors, from_pages, to_pages)
    if st:
        ctx._check(st)


@dataclass
class Samples:
    """Outputs of mt_sample; one that is set to None is left out."""
    ids: Optional[torch.Tensor]              # int32 [R]
    logprobs: Optional[torch.Tensor]         # float32 [R]
    kept: Optional[torch.Tensor]             # int32 [R]
    scratch: Optional[torch.Tensor] = None   # uint8; not used: a call needs none


def alloc_samples(rows: int, classes: int, device="cuda:0") -> Samples:
    """Outputs of mt_sample for so many rows and classes."""
    ints = lambda: torch.empty(rows, dtype=torch.int32, device=device)  # noqa: E731
    return Samples(ints(), torch.empty(rows, dtype=torch.float32, device=device), ints(), torch.zeros(B.sample_scratch(rows, classes), dtype=torch.uint8, device=device))


def sample(ctx: B.Context, logits: torch.Tensor, uniform: torch.Tensor, out: Samples, temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
           top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None, n_classes: Optional[torch.Tensor] = None, allowed: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> Samples:
    """mt_sample on the given (or current) stream: one class for every row of logits, from the random numbers uniform (float32 [rows], in [0, 1)) and the rows' settings: temperature,
    top_p, min_p float32 [rows], top_k int32 [rows].  n_classes, allowed: as in score.  Forward only."""
    st = (_answers or answers()).sample(*_where(ctx, stream), logits, uniform, temperature, top_k, top_p, min_p, n_classes, allowed, out.ids, out.logprobs, out.kept, out.scratch)
    if st:
        ctx._check(st)
    return out
