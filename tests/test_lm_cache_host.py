"""Host logic of the calls on language models' caches: argument checks.  No GPU, no compute."""
import ctypes

import numpy as np
import pytest

import lm_cache_common as lc
import lm_common as lm
import paper_1901_06887_amd as mt
from paper_1901_06887_amd import binding as B
from test_lm_host import host_ctx, refused


def cache(**kw):
    c = B.mt_kv_cache()
    base = dict(k=64, v=64, table=64, lengths=64, refs=64, work=64, page_stride=2 * 32 * 64, layer_stride=2 * 32 * 64 * 10, table_stride=7, work_bytes=1 << 20,
                dtype=B.MT_BF16, layers=3, n_pages=10, heads=2, page_tokens=32, head_dim=64, seqs=5, table_width=7)
    for k, v in {**base, **kw}.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    b = B.mt_kv_batch()
    for k, v in {**dict(rows=5, n_seqs=5, max_new=1), **kw}.items():
        setattr(b, k, v)
    return b


KV8 = dict(dtype=B.MT_KV8, k_scales=64, v_scales=64, scales_page_stride=64, scales_layer_stride=640)
BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(table=None), 1), (dict(lengths=None), 1), (dict(dtype=B.MT_MX8), 5), (dict(dtype=4), 5), (dict(k_scales=64), 1), (dict(v_scales=64), 1),
              (dict(KV8, k_scales=None), 1), (dict(KV8, v_scales=None), 1), (dict(layers=0), 1), (dict(n_pages=0), 1), (dict(heads=0), 1), (dict(seqs=0), 1), (dict(table_width=0), 1),
              (dict(page_tokens=8), 5), (dict(page_tokens=48), 5), (dict(page_tokens=512), 5), (dict(page_tokens=0), 5), (dict(head_dim=0), 5), (dict(head_dim=72), 5), (dict(head_dim=272), 5),
              (dict(seqs=16385), 5), (dict(table_width=131073, table_stride=131073), 5), (dict(n_pages=1 << 31), 5), (dict(k=72), 1), (dict(v=66), 1), (dict(page_stride=4097), 1),
              (dict(layer_stride=40961), 1), (dict(KV8, k_scales=65), 1), (dict(KV8, scales_page_stride=65), 1), (dict(page_stride=4088), 1), (dict(layer_stride=4088), 1),
              (dict(layer_stride=4096 * 9), 1), (dict(page_stride=8192), 1), (dict(KV8, scales_layer_stride=576), 1), (dict(table_stride=6), 1)]
GOOD_CACHES = [dict(), KV8, dict(page_stride=3 * 4096, layer_stride=4096), dict(layers=1, layer_stride=0), dict(n_pages=1, page_stride=0), dict(dtype=B.MT_F32), dict(page_stride=1 << 60, layer_stride=4096)]


def write_args(**kw):
    a = B.mt_kv_write_args()
    for k, v in {**dict(k=64, v=64, k_stride=128, v_stride=128, dtype=B.MT_BF16, layer=2), **kw}.items():
        setattr(a, k, v)
    return a


def attend_args(**kw):
    a = B.mt_attend_args()
    base = dict(q=64, out=64, scratch=64, scratch_bytes=1 << 30, q_stride=6 * 64, out_stride=6 * 64, q_heads=6, dtype=B.MT_BF16, layer=2, scale=0.125)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def test_struct_layouts():
    assert ctypes.sizeof(B.mt_kv_cache) == 8 * 8 + 6 * 8 + 8 * 4
    assert ctypes.sizeof(B.mt_kv_batch) == 2 * 8 + 4 * 4
    assert ctypes.sizeof(B.mt_kv_write_args) == 4 * 8 + 2 * 4
    assert ctypes.sizeof(B.mt_attend_args) == 7 * 8 + 6 * 4
    assert ctypes.sizeof(B.mt_sample_args) == 12 * 8 + 3 * 8 + 4 * 4


def test_caches_that_are_refused():
    c = host_ctx()
    rows = lambda kw: B.MT_F32 if kw.get("dtype") == B.MT_F32 else B.MT_BF16  # noqa: E731
    for kw, status in [*BAD_CACHES, *((kw, 7) for kw in GOOD_CACHES)]:
        k = cache(**kw)
        refused(status, c.kv_write, 0, k, batch(), write_args(dtype=rows(kw), layer=0))
        refused(status, c.attend, 0, k, batch(), attend_args(dtype=rows(kw), layer=0))
        for f, args in ((c.kv_grow, (64, 64, 3)), (c.kv_fork, (64, 64, 3)), (c.kv_free, (64, 3)), (c.kv_compact, ()), (c.kv_copy, (64, 64, 3))):
            refused(status, f, 0, k, *args)
    c.close()


def test_rows_that_are_refused():
    c = host_ctx()
    for call, args, width in ((c.kv_write, write_args, ("k_stride", 127)), (c.attend, attend_args, ("q_stride", 6 * 64 - 1))):
        for kw, status in ((dict(dtype=B.MT_F32), 5), (dict(dtype=B.MT_MX8), 5), (dict(layer=3), 1), ({width[0]: width[1]}, 1)):
            refused(status, call, 0, cache(), batch(), args(**kw))
        refused(7, call, 0, cache(**KV8), batch(), args(dtype=B.MT_F32))
        for kw, status in ((dict(rows=4), 1), (dict(n_seqs=6, rows=6), 1), (dict(max_new=0), 1), (dict(rows=9, first_row=64), 7), (dict(n_seqs=6, rows=6, seqs=64), 7), (dict(rows=0, n_seqs=0), 7),
                           (dict(rows=0, first_row=64), 7), (dict(n_seqs=(1 << 20) + 1, rows=(1 << 20) + 1, seqs=64), 5)):
            refused(status, call, 0, cache(), batch(**kw), args())
    refused(1, c.kv_write, 0, cache(), batch(), write_args(k=None))
    refused(1, c.kv_write, 0, cache(), batch(), write_args(v=None))
    refused(1, c.kv_write, 0, cache(), batch(), write_args(v_stride=127))
    for kw, status in ((dict(q=None), 1), (dict(out=None), 1), (dict(out_stride=383), 1), (dict(q_heads=0), 1), (dict(q_heads=5), 1), (dict(q_heads=65536, q_stride=1 << 30, out_stride=1 << 30), 5),
                       (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(scale=2e38), 1), (dict(scale=-1e38), 7)):
        refused(status, c.attend, 0, cache(), batch(), attend_args(**kw))
    lib = B.load_library()
    k, b, w, a = cache(), batch(), write_args(), attend_args()
    for f, args in ((lib.mt_kv_write, w), (lib.mt_attend, a)):
        assert f(None, None, ctypes.byref(k), ctypes.byref(b), ctypes.byref(args)) == 1
        assert f(c._h, None, None, ctypes.byref(b), ctypes.byref(args)) == 1
        assert f(c._h, None, ctypes.byref(k), None, ctypes.byref(args)) == 1
        assert f(c._h, None, ctypes.byref(k), ctypes.byref(b), None) == 1
    c.close()


def test_attend_needs_its_scratch():
    c = host_ctx()
    k = cache(table_width=4096, table_stride=4096, n_pages=1 << 20, layers=1)
    need = mt.attend_scratch(k, 2, 6)
    if need:
        for kw in (dict(scratch=None), dict(scratch_bytes=need - 1), dict(scratch=72)):
            assert "scratch" in refused(1, c.attend, 0, k, batch(rows=2, n_seqs=2), attend_args(**dict(dict(scratch_bytes=need, layer=0), **kw)))
        refused(7, c.attend, 0, k, batch(rows=2, n_seqs=2), attend_args(scratch_bytes=need, layer=0))
    refused(1, mt.attend_scratch, k, 2, 5)
    refused(1, mt.attend_scratch, k, 2, 0)
    c.close()


def test_pages_that_are_refused():
    c = host_ctx()
    need = mt.kv_work(10, 5)
    for f, args in ((c.kv_grow, (None, 64)), (c.kv_fork, (64, 64)), (c.kv_free, (64,)), (c.kv_copy, (64, 64))):
        refused(7, f, 0, cache(), *args, 5)
        refused(7, f, 0, cache(), *args, 0)
        refused(7 if f == c.kv_copy else 1, f, 0, cache(), *args, 6)
        for kw in (dict(refs=None), dict(work=None), dict(work=72), dict(work_bytes=need - 1)):
            refused(1, f, 0, cache(**kw), *args, 3)
        refused(7, f, 0, cache(work_bytes=need), *args, 3)
    for f, args in ((c.kv_grow, (64, None)), (c.kv_fork, (None, 64)), (c.kv_fork, (64, None)), (c.kv_free, (None,)), (c.kv_copy, (None, 64)), (c.kv_copy, (64, None))):
        refused(1, f, 0, cache(), *args, 1)
    refused(1, c.kv_compact, 0, cache(refs=None))
    for a in ((0, 5, 1), (5, 0, 1), (5, 16385, 5), (1 << 31, 5, 5)):
        refused(a[2], mt.kv_work, a[0], a[1])
    c.close()


def sample_args(**kw):
    a = B.mt_sample_args()
    for k, v in {**dict(logits=64, uniform=64, ids=64, scratch=64, scratch_bytes=1 << 30, row_stride=100, rows=7, classes=100, dtype=B.MT_F32), **kw}.items():
        setattr(a, k, v)
    return a


def test_sample_refuses():
    c = host_ctx()
    for kw, status in ((dict(logits=None), 1), (dict(uniform=None), 1), (dict(ids=None), 1), (dict(classes=0), 1), (dict(row_stride=99), 1), (dict(dtype=2), 5), (dict(allowed=64, allowed_stride=3), 1),
                       (dict(classes=(1 << 20) + 1, row_stride=1 << 21), 5), (dict(ids=None, kept=64), 7), (dict(rows=0, logits=None), 7), ({}, 7)):
        refused(status, c.sample, 0, sample_args(**kw))
    big = dict(classes=131072, row_stride=131072, rows=1)
    need = mt.sample_scratch(1, 131072)
    if need:
        for kw in (dict(scratch=None), dict(scratch_bytes=need - 1), dict(scratch=72)):
            assert "scratch" in refused(1, c.sample, 0, sample_args(**big, **kw))
    refused(1, mt.sample_scratch, 5, 0)
    refused(5, mt.sample_scratch, 5, (1 << 20) + 1)
    lib = B.load_library()
    assert lib.mt_sample(c._h, None, None) == 1 and lib.mt_sample(None, None, ctypes.byref(sample_args())) == 1
    c.close()


def test_calls_on_tensors_refuse_what_is_no_tensor_on_the_device():
    import torch
    c = host_ctx()
    k = mt.alloc_kv(4, 16, 2, 32, 3, 2, device="cpu")
    x, ints = torch.zeros(3, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    calls = mt.torch_io.answers()
    for f, args in ((calls.kv_write, (x, x, None, None, 1, 0)), (calls.attend, (x, x, None, None, 1, 0, 0, 0, None, None, None)), (calls.kv_grow, (None, ints, None)), (calls.kv_fork, (ints, ints, None)),
                    (calls.kv_free, (ints,)), (calls.kv_compact, (None,)), (calls.kv_copy, (ints, ints))):
        for spec, tensors in ((k.spec, k._tensors), (None, k._tensors), (k.spec, None), (b"short", k._tensors), (k.spec, (1, 2))):
            with pytest.raises(ValueError, match="cache"):
                f(c._h.value, 0, 0, spec, tensors, *args)
        with pytest.raises(TypeError):
            f(c._h.value, 0, 0, k.spec, k._tensors, *args, None)
        if args[0] is not None:
            with pytest.raises(ValueError):
                f(c._h.value, 0, 0, k.spec, (), *args)
    with pytest.raises(ValueError):
        calls.sample(c._h.value, 0, 0, torch.zeros(2, 8), torch.zeros(2), *[None] * 9, ints)
    with pytest.raises(ValueError):
        mt.alloc_kv(4, 16, 2, 32, 3, 2, dtype=mt.MT_MX8, device="cpu")
    c.close()


def test_the_oracle_of_8_bits():
    """Nearest values by trying all of them."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 3, 32)) * 10.0 ** rng.integers(-6, 6, (50, 3, 1))
    x[3, 1] = 0
    q, e = lc.in_8_bits(x)
    all_values = lm.e4m3(np.arange(256))
    scaled = x / lm.e8m0(e)[..., None]
    best = np.nanmin(np.abs(scaled[..., None] - all_values), axis=-1)
    assert np.array_equal(np.abs(lm.e4m3(q) - scaled), best)
    most = np.abs(x).max(-1)
    assert np.all(most <= 448 * lm.e8m0(e)) and np.all((most > 448 * lm.e8m0(e) / 2) | (most == 0)) and e[3, 1] == 127


def test_the_oracle_of_the_next_class():
    """A class is drawn as often as its share says, over a fine grid of random numbers; settings keep what they should."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal(12).astype(np.float32).astype(np.float64)
    for kw in (dict(), dict(temperature=0.5), dict(top_k=4), dict(top_p=0.7), dict(min_p=0.3), dict(top_k=6, top_p=0.8, min_p=0.1), dict(n=7), dict(temperature=0.0), dict(allowed=np.array([0x0f6], dtype=np.uint32))):
        picks = [lc.sampled(x, u, **kw) for u in (np.arange(4000) + 0.5) / 4000]
        counts = np.bincount([p[0] for p in picks], minlength=12) / 4000
        for c in range(12):
            lp = [p[1] for p in picks if p[0] == c]
            if lp:
                assert abs(np.exp(lp[0]) - counts[c]) <= 1 / 4000
        assert len({p[2] for p in picks}) == 1 and (counts > 0).sum() <= picks[0][2]
    assert lc.sampled(x, 0.5, top_k=1)[0] == x.argmax() and lc.sampled(x, 0.5, top_p=0.0)[2] == 1 and lc.sampled(x, 0.5, temperature=-1.0)[2] == -1


def test_the_oracle_of_books():
    b = lc.Books(8, 4, 4, 5)
    assert b.grow([0, 1, 0, 9], [6, 4, 1, 1]) == [1, 1, 0, 0] and b.table[:2] == [[0, 1], [2]]
    assert b.fork([0, 0, 1], [2, 3, 2]) == [1, 1, 0] and b.table[2] == [0, 3] and b.table[3] == [0, 4] and b.refs[0] == 3 and b.contents[3] == b.contents[4] == 1
    assert b.grow([1, 2, 3], [8, 12, 2]) == [1, 0, 1] and b.grow([1], [9]) == [0]
    b.free([0, 0])
    assert b.refs[0] == 2 and b.refs[1] == 0
    assert b.compact() == 6 and b.table[1] == [2, 5, 1]
