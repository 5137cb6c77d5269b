"""Host logic of the operators behind language models' answers: argument checks, matrices in a host-only context's arena.  No GPU, no compute."""
import ctypes

import numpy as np
import pytest

import lm_common as lm
import paper_1901_06887_amd as mt
from paper_1901_06887_amd import binding as B


def host_ctx(arena=1 << 20, cache=False):
    return B.Context(2, 16, 64, 16, arena, B.MT_F32, device=-1, cache=cache)


def refused(status, f, *a):
    with pytest.raises(B.MtError) as e:
        f(*a)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def test_struct_layouts():
    assert ctypes.sizeof(B.mt_norm_args) == 8 * 8 + 7 * 8 + 6 * 4
    assert ctypes.sizeof(B.mt_row_group) == 12
    assert ctypes.sizeof(B.mt_linear4_args) == 3 * 8 + 3 * 8 + 4 * 4
    assert ctypes.sizeof(B.mt_score_args) == 10 * 8 + 3 * 8 + 6 * 4


def test_matrices_take_and_return_arena():
    c = host_ctx()
    rng = np.random.default_rng(0)
    tiles = lambda n, k: -(-n // 16) * -(-k // 128) * 1088  # noqa: E731
    sizes = [(1, 1), (16, 128), (17, 129), (333, 301), (100, 4096)]
    numbers, used = [], 0
    for n, k in sizes:
        codes, scales, _ = lm.random_matrix(rng, n, k)
        numbers.append(c.register_matrix4(n, k, codes, scales, np.zeros(n) if n % 2 else None))
        want = (tiles(n, k) + 4 * n + 255) // 256 * 256
        assert mt.matrix4_footprint(n, k) == want
        used += want
        assert c.stats()["arena_used"] == used
    assert numbers == [0, 1, 2, 3, 4]
    c.unregister_matrix4(2)
    used -= mt.matrix4_footprint(17, 129)
    assert c.stats()["arena_used"] == used
    refused(3, c.unregister_matrix4, 2)
    refused(3, c.unregister_matrix4, 5)
    codes, scales, _ = lm.random_matrix(rng, 3, 5)
    assert c.register_matrix4(3, 5, codes, scales) == 2
    codes, scales, _ = lm.random_matrix(rng, 2000, 2000)
    before = c.stats()["arena_used"]
    refused(2, c.register_matrix4, 2000, 2000, codes, scales)
    codes, scales, _ = lm.random_matrix(rng, 1000, 1000)
    refused(2, c.register_matrix4, 1000, 1600, *lm.random_matrix(rng, 1000, 1600)[:2])
    assert c.stats()["arena_used"] == before and c.stats()["n_tenants"] == 0
    c.close()


def test_models_of_a_cache_give_way_to_matrices():
    c = host_ctx(arena=1 << 18, cache=True)
    specs = [B.layer_spec(B.MT_FC, B.MT_ACT_NONE, 64, 10)]
    c.register_model(0, specs, [np.zeros((10, 64), np.float32)], [None])
    rng = np.random.default_rng(0)
    n = 16
    k = ((1 << 18) - 256) // 1088 * 128
    c.register_matrix4(n, k, *lm.random_matrix(rng, n, k)[:2])
    assert c.cache_stats()["evictions"] == 1 and c.tenant_account(0)["resident"] == 0
    refused(2, c.prefetch, [0])                      # a matrix does not give way to a model
    c.unregister_matrix4(0)
    c.prefetch([0])
    assert c.tenant_account(0)["resident"] == 1
    c.close()


def test_registration_refuses():
    c = host_ctx()
    rng = np.random.default_rng(0)
    codes, scales, _ = lm.random_matrix(rng, 4, 64)
    for bad in (0, 26, 228, 255):
        s = scales.copy()
        s[2, 1] = bad
        refused(5, c.register_matrix4, 4, 64, codes, s)
    with pytest.raises(ValueError):
        c.register_matrix4(4, 65, codes, scales)
    with pytest.raises(ValueError):
        c.register_matrix4(4, 64, codes, scales, np.zeros(5))
    lib, n = B.load_library(), ctypes.c_uint32()
    p = codes.ctypes.data
    for args in ((4, 64, None, p, None, n), (4, 64, p, None, None, n), (0, 64, p, p, None, n), (4, 0, p, p, None, n)):
        assert lib.mt_register_matrix4(c._h, *args[:5], ctypes.byref(args[5])) == 1
    assert lib.mt_register_matrix4(c._h, 4, 64, p, p, None, None) == 1
    assert lib.mt_register_matrix4(None, 4, 64, p, p, None, ctypes.byref(n)) == 1
    assert lib.mt_register_matrix4(c._h, (1 << 24) + 1, 64, p, p, None, ctypes.byref(n)) == 5
    for a in ((0, 5, 1), (5, 0, 1), (1 << 25, 5, 5)):
        refused(a[2], mt.matrix4_footprint, a[0], a[1])
    assert c.stats()["arena_used"] == 0
    c.close()


def norm_args(**kw):
    a = B.mt_norm_args()
    base = dict(x=64, y=64, x_stride=100, y_stride=100, rows=3, width=100, dtype=B.MT_F32, eps=1e-6)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def test_add_norm_refuses():
    c = host_ctx()
    for kw, status in ((dict(x=None), 1), (dict(y=None), 1), (dict(width=0), 1), (dict(x_stride=99), 1), (dict(y_stride=99), 1), (dict(dtype=2), 5), (dict(dtype=9), 5),
                       (dict(residual=64, residual_stride=5), 1), (dict(gain=64, gain_stride=99, n_gains=1), 1), (dict(gain=64, gain_stride=100, n_gains=0), 1),
                       (dict(gain_ids=64), 1), (dict(y8=64, y8_stride=100), 1), (dict(y8_scales=64, y8_scales_stride=4), 1), (dict(y8=64, y8_stride=100, y8_scales=64, y8_scales_stride=3), 1),
                       (dict(sum=64, sum_stride=1), 1), (dict(eps=-1e-6), 1), (dict(eps=float("inf")), 1), ({}, 7)):
        refused(status, c.add_norm, 0, norm_args(**kw))
    wide = (1 << 24) + 1
    refused(5, c.add_norm, 0, norm_args(width=wide, x_stride=wide, y_stride=wide))
    assert B.load_library().mt_add_norm(c._h, None, None) == 1 and B.load_library().mt_add_norm(None, None, ctypes.byref(norm_args())) == 1
    c.close()


def linear_args(**kw):
    a = B.mt_linear4_args()
    base = dict(x=64, y=64, x_stride=64, y_stride=8, rows=10, x_dtype=B.MT_F32, y_dtype=B.MT_F32, act=0)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def test_linear4_refuses():
    c = host_ctx()
    rng = np.random.default_rng(0)
    m = c.register_matrix4(8, 64, *lm.random_matrix(rng, 8, 64)[:2])
    one = mt.row_groups([(m, 0, 10)])
    for kw, status in ((dict(x=None), 1), (dict(y=None), 1), (dict(x_dtype=3), 5), (dict(y_dtype=2), 5), (dict(act=3), 5), (dict(x_stride=63), 1), (dict(y_stride=7), 1),
                       (dict(x_dtype=B.MT_MX8), 1), (dict(x_scales=64), 1), (dict(x_dtype=B.MT_MX8, x_scales=64, x_scales_stride=1), 1), (dict(rows=9), 1), ({}, 7)):
        refused(status, c.linear4, 0, linear_args(**kw), one)
    for groups, status in (([(m, 0, 11)], 1), ([(m, 3, 1), (m, 2, 1)], 1), ([(m, 0, 4), (m, 3, 1)], 1), ([(m + 1, 0, 1)], 3), ([(m, 0, 1), (77, 1, 1)], 3), ([(m, 4294967295, 4294967295)], 1),
                           ([(m, 0, 4), (m, 4, 6)], 7)):
        refused(status, c.linear4, 0, linear_args(), mt.row_groups(groups))
    lib = B.load_library()
    assert lib.mt_linear4(c._h, None, None, one, 1) == 1 and lib.mt_linear4(c._h, None, ctypes.byref(linear_args()), None, 1) == 1
    assert lib.mt_linear4(None, None, ctypes.byref(linear_args()), one, 1) == 1
    c.close()


def score_args(**kw):
    a = B.mt_score_args()
    base = dict(logits=64, entropy=64, row_stride=100, rows=2000, classes=100, dtype=B.MT_F32, temperature=1.0)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def test_score_refuses():
    c = host_ctx()
    for kw, status in ((dict(logits=None), 1), (dict(entropy=None), 1), (dict(classes=0), 1), (dict(row_stride=99), 1), (dict(dtype=2), 5), (dict(temperature=0.0), 1),
                       (dict(temperature=-2.0), 1), (dict(temperature=float("nan")), 1), (dict(temperature=float("inf")), 1), (dict(given=64), 1), (dict(n_given=1), 1),
                       (dict(given_ranks=64), 1), (dict(n_given=17, given=64), 1), (dict(top=33, top_ids=64), 1), (dict(top_ids=64), 1), (dict(allowed=64, allowed_stride=3), 1),
                       (dict(classes=1 << 31, row_stride=1 << 31), 1), ({}, 7)):
        refused(status, c.score, 0, score_args(**kw))
    need = mt.score_scratch(1, 131072, 1, 20)
    if need:
        big = dict(rows=1, classes=131072, row_stride=131072, given=64, n_given=1, given_ranks=64, top=20, top_ids=64)
        for kw in (dict(), dict(scratch=64), dict(scratch=64, scratch_bytes=need - 1), dict(scratch=72, scratch_bytes=need)):
            assert "scratch" in refused(1, c.score, 0, score_args(**big, **kw))
        refused(7, c.score, 0, score_args(**big, scratch=64, scratch_bytes=need))
    for a in ((1, 0, 0, 0), (1, 5, 17, 0), (1, 5, 0, 33)):
        refused(1, mt.score_scratch, *a)
    # what is enough for more rows or classes is enough for fewer
    for top in (0, 20):
        for rows in (1, 2, 5, 40, 300, 2000):
            assert mt.score_scratch(rows, 2 ** 31 - 1, 1, top) >= max(mt.score_scratch(rows, n, 1, top) for n in (1, 100, 3000, 65001, 10 ** 6))
    lib = B.load_library()
    assert lib.mt_score(c._h, None, None) == 1 and lib.mt_score(None, None, ctypes.byref(score_args())) == 1
    c.close()


def test_calls_on_tensors_refuse_what_is_no_tensor_on_the_device():
    """Without a GPU no call goes through: every operand is looked at before anything is dereferenced."""
    import torch
    c = host_ctx()
    x = torch.zeros(2, 8)
    calls = mt.torch_io.answers()
    for f, args in ((calls.add_norm, (x, None, None, None, 1e-6, None, x, None, None)), (calls.add_norm, (3, None, None, None, 1e-6, None, x, None, None)),
                    (calls.linear4, (mt.row_groups([(0, 0, 2)]), x, x, None, 0)), (calls.linear4, (None, x.half(), x, None, 0)),
                    (calls.score, (x, None, None, None, 1.0, None, None, x[0], None, None, x)), (calls.score, (x[0], None, None, None, 1.0, None, None, x[0], None, None, x))):
        with pytest.raises(ValueError):
            f(c._h.value, 0, 0, *args)
        with pytest.raises(TypeError):
            f(c._h.value, 0, 0, *args, None)
    c.close()


def test_linear4_of_narrow_rows_refuses():
    """Strides wide enough for the matrix, columns too few: a slice of a padded buffer.  Groups of 0 rows touch nothing."""
    c = host_ctx()
    rng = np.random.default_rng(0)
    m = c.register_matrix4(8, 64, *lm.random_matrix(rng, 8, 64)[:2])
    wide = c.register_matrix4(9, 65, *lm.random_matrix(rng, 9, 65)[:2])
    lib = B.load_library()
    args = linear_args(x_stride=96, y_stride=32)
    for groups, x_width, y_width, status in (([(m, 0, 10)], 63, 8, 1), ([(m, 0, 10)], 64, 7, 1), ([(m, 0, 10)], 64, 8, 7), ([(m, 0, 5), (wide, 5, 1)], 64, 9, 1),
                                             ([(m, 0, 5), (wide, 5, 1)], 65, 8, 1), ([(m, 0, 5), (wide, 5, 1)], 65, 9, 7), ([(m, 0, 5), (wide, 5, 0)], 64, 8, 7)):
        g = mt.row_groups(groups)
        assert lib.mt_linear4_within(c._h, None, ctypes.byref(args), g, len(g), x_width, y_width) == status, (groups, x_width, y_width)
    assert lib.mt_linear4_within(None, None, ctypes.byref(args), None, 0, 64, 8) == 1
    c.close()


def test_score_refuses_temperatures_below_the_normal_range():
    c = host_ctx()
    for t in (2.0 ** -126 * (1 - 2.0 ** -23), 6e-39, 4e-39, 3e-39):
        refused(1, c.score, 0, score_args(temperature=t))
    for t in (2.0 ** -126, 3.4e38):
        refused(7, c.score, 0, score_args(temperature=t))
    c.close()


def test_forms_of_linear4_by_sizes():
    """The rule on 256 compute units, on both sides of its lines: (rows, out, in) of every group; outputs and rows of a workgroup, rows through LDS."""
    for kind, groups, want in ((B.MT_BF16, [(1, 1024, 1024)], (16, 16, False)), (B.MT_BF16, [(1, 65536, 4096)], (64, 16, False)), (B.MT_BF16, [(512, 4096, 4096)], (128, 64, True)),
                               (B.MT_MX8, [(50, 4096, 4096)] * 8, (128, 64, True)), (B.MT_BF16, [(64, 4096, 4096)] * 4, (128, 64, True)), (B.MT_BF16, [(64, 4096, 4096)] * 3, (64, 16, False)),
                               (B.MT_BF16, [(24, 2064, 1100)] * 8, (128, 32, True)), (B.MT_BF16, [(16, 2064, 1100)] * 16, (64, 16, False)), (B.MT_F32, [(16, 2064, 1100)] * 16, (128, 16, True)),
                               (B.MT_F32, [(64, 4096, 1023)] * 2, (64, 16, False)), (B.MT_F32, [(64, 4096, 1024)] * 2, (128, 16, True)), (B.MT_F32, [(0, 4096, 4096), (1, 100, 64)], (16, 16, False))):
        assert mt.debug_linear4_shape(groups, 256, kind) == dict(zip(("outputs", "rows", "through_lds"), want)), (kind, groups)
