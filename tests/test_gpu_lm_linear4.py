"""mt_linear4 against the products of the dequantised weights in 64 bits."""
from math import erf

import numpy as np
import pytest
import torch

import lm_common as lm
import paper_1901_06887_amd as mt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def context(arena=64 << 20):
    return mt.Context(1, 1, 64, 1, arena, mt.MT_BF16, 0)


def rows_in(rng, kind, rows, k, stride, offset=0):
    """(tensor, scales or None, values) of rows whose buffer holds NaN everywhere else."""
    if kind == "mx8":
        codes = rng.integers(0, 256, (rows, k), dtype=np.uint8)
        codes[(codes & 127) == 127] = 0
        e = rng.integers(120, 130, (rows, -(-k // 32)), dtype=np.uint8)
        buf = torch.full((offset + rows * stride + 16,), 127, dtype=torch.uint8, device="cuda")
        v = buf[offset:offset + rows * stride].view(rows, stride)[:, :k]
        v.copy_(torch.from_numpy(codes))
        n = e.shape[1]
        ebuf = torch.full((rows * (n + 3) + 4,), 255, dtype=torch.uint8, device="cuda")
        ev = ebuf[:rows * (n + 3)].view(rows, n + 3)[:, :n]
        ev.copy_(torch.from_numpy(e))
        return v.view(torch.float8_e4m3fn), ev.view(torch.float8_e8m0fnu), lm.e4m3(codes) * lm.spread(lm.e8m0(e), k)
    buf = torch.full((offset + rows * stride + 16,), float("nan"), dtype=DT[kind], device="cuda")
    v = buf[offset:offset + rows * stride].view(rows, stride)[:, :k]
    v.copy_(torch.from_numpy(rng.standard_normal((rows, k))))
    return v, None, v.double().cpu().numpy()


def check(y, x, w, bias, act, x_kind, y_kind):
    """Products are exact, a sum has at most one rounding for every 8 of the fan-in (three parts of fp32 rows: thrice), and some for joining parts, the
    bias and the activation."""
    K = x.shape[1]
    ref = x @ w.T + (0.0 if bias is None else bias.astype(np.float64))
    size = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    bound = (K / 8 * (3 if x_kind == "f32" else 1) + 40) * 2.0 ** -24 * size
    if act == mt.MT_ACT_RELU:
        ref = np.maximum(ref, 0)
    elif act == mt.MT_ACT_GELU:
        ref = 0.5 * ref * (1 + np.vectorize(erf)(ref * np.sqrt(0.5)))
        bound = 1.13 * bound + 2e-6 * np.abs(ref) + 1e-7
    bound = bound + (2.0 ** -8 if y_kind == "bf16" else 2.0 ** -23) * (np.abs(ref) + bound)
    off = np.abs(y - ref)
    assert np.all(off <= bound), (np.max(off / np.maximum(bound, 1e-300)), np.unravel_index(np.argmax(off - bound), off.shape))


def call(ctx, groups, x, scales, rows, n, y_kind, act, stride=None):
    stride = stride or n + 5
    buf = torch.full((rows * stride + 8,), 7.0, dtype=DT[y_kind], device="cuda")
    y = buf[:rows * stride].view(rows, stride)[:, :n]
    mt.linear4(ctx, mt.row_groups(groups), x, y, x_scales=scales, act=act)
    torch.cuda.synchronize()
    assert torch.all(buf[:rows * stride].view(rows, stride)[:, n:] == 7.0) and torch.all(buf[rows * stride:] == 7.0)
    return y.double().cpu().numpy()


SHAPES = [(1, 1), (1, 16), (2, 10), (31, 15), (32, 17), (33, 64), (96, 65), (127, 1), (128, 16), (129, 33), (256, 130), (301, 333), (512, 48), (784, 1024), (1000, 100), (1025, 257),
          (2048, 96), (4100, 40)]


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("y_kind", ["bf16", "f32"])
@pytest.mark.parametrize("k,n", SHAPES)
def test_sizes(x_kind, y_kind, k, n):
    rng = np.random.default_rng(1000 * k + n)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, n, k)
    bias = rng.standard_normal(n).astype(np.float32)
    m = [ctx.register_matrix4(n, k, codes, scales, bias), ctx.register_matrix4(n, k, codes, scales)]
    for i, rows in enumerate((1, 3, 16, 17, 33, 64, 65, 130)):
        x, e, v = rows_in(rng, x_kind, rows, k, k + (0, 1, 8)[i % 3], i % 4)
        act = (mt.MT_ACT_NONE, mt.MT_ACT_RELU, mt.MT_ACT_GELU)[i % 3]
        y = call(ctx, [(m[i % 2], 0, rows)], x, e, rows, n, y_kind, act)
        check(y, v, w, bias if i % 2 == 0 else None, act, x_kind, y_kind)
    ctx.close()


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("rows,N,K", [(1, 500, 1024), (3, 8192, 1030), (20, 2000, 257), (130, 8192, 1024), (130, 8192, 1100), (40, 8192, 1024)])
def test_every_bit_of_a_value_arrives(x_kind, rows, N, K):
    """Matrices of one power of two to an output: no sum rounds, so every output is that column times it, to the last bit."""
    rng = np.random.default_rng(rows + K)
    ctx = context()
    w, at = np.zeros((N, K)), rng.integers(0, K, N)
    codes, which = np.zeros((N, K + K % 2), dtype=np.uint8), rng.integers(0, 8, N)
    codes[np.arange(N), at] = np.array([1, 2, 4, 6, 9, 10, 12, 14])[which]                 # +-0.5, 1, 2, 4
    w[np.arange(N), at] = lm.E2M1[codes[np.arange(N), at]]
    m = ctx.register_matrix4(N, K, codes[:, 0::2] | codes[:, 1::2] << 4, np.full((N, -(-K // 32)), 127, dtype=np.uint8))
    x, e, v = rows_in(rng, x_kind, rows, K, K, 0)
    y = call(ctx, [(m, 0, rows)], x, e, rows, N, "f32", mt.MT_ACT_NONE)
    assert np.array_equal(y, v[:, at] * w[np.arange(N), at])
    ctx.close()


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("lo,hi", [(1, 1), (1, 3), (0, 40), (60, 150)])
def test_tenants_of_all_sizes_in_one_call(x_kind, lo, hi):
    """More groups than a launch holds, matrices that all differ, rows that belong to nobody, a tenant with two groups."""
    rng = np.random.default_rng(hi)
    ctx = context()
    K, N, T = 400, 300, 70 if hi < 100 else 9
    mats, at, groups = [], 2, []
    for t in range(T):
        k, n = int(rng.integers(1, K + 1)), int(rng.integers(1, N + 1))
        codes, scales, w = lm.random_matrix(rng, n, k)
        bias = rng.standard_normal(n).astype(np.float32) if t % 2 else None
        mats.append((ctx.register_matrix4(n, k, codes, scales, bias), k, n, w, bias))
    for t in list(range(T)) + [3]:
        rows = int(rng.integers(lo, hi + 1))
        groups.append((t, at, rows))
        at += rows + (t % 5 == 0)
    x, e, v = rows_in(rng, x_kind, at, K, K + 1, 1)
    y = torch.full((at, N), 7.0, device="cuda")
    mt.linear4(ctx, mt.row_groups([(mats[t][0], a, r) for t, a, r in groups]), x, y, x_scales=e)
    y = y.double().cpu().numpy()
    touched = np.zeros(at, dtype=bool)
    for t, a, r in groups:
        _, k, n, w, bias = mats[t]
        if r:
            check(y[a:a + r, :n], v[a:a + r, :k], w, bias, mt.MT_ACT_NONE, x_kind, "f32")
        assert np.all(y[a:a + r, n:] == 7.0)
        touched[a:a + r] = True
    assert np.all(y[~touched] == 7.0)
    ctx.close()


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("rows,k,n", [(200, 1024, 600), (300, 520, 1100), (513, 4096, 272), (1, 4096, 5000), (16, 2048, 4100), (40, 8200, 1000)])
def test_larger_products(x_kind, rows, k, n):
    rng = np.random.default_rng(rows + k)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, n, k)
    m = ctx.register_matrix4(n, k, codes, scales)
    x, e, v = rows_in(rng, x_kind, rows, k, k)
    for y_kind in ("bf16", "f32"):
        y = torch.empty(rows, n, dtype=DT[y_kind], device="cuda")
        mt.linear4(ctx, mt.row_groups([(m, 0, rows)]), x, y, x_scales=e)
        some = rng.permutation(rows)[:24]
        check(y.double().cpu().numpy()[some], v[some], w, None, mt.MT_ACT_NONE, x_kind, y_kind)
    ctx.close()


def test_every_code_and_scale_is_exact():
    """One weight per output against one value per row: the product itself."""
    ctx = context()
    n = 16 * 8
    codes = np.zeros((n, 16), dtype=np.uint8)
    scales = np.full((n, 1), 127, dtype=np.uint8)
    for i, s in enumerate((27, 60, 126, 127, 128, 190, 226, 227)):
        codes[16 * i:16 * i + 16, 3] = np.arange(16) << 4          # column 7
        scales[16 * i:16 * i + 16] = s
    w = lm.E2M1[codes[:, 3] >> 4] * lm.e8m0(scales[:, 0])
    m = ctx.register_matrix4(n, 32, codes, scales)
    vals = np.array([1 + 2.0 ** -23, -(2 - 2.0 ** -23), 3.0e-3, 1.1754944e-20, 65537.0, 1 / 3], dtype=np.float32)
    x = torch.zeros(len(vals), 32, device="cuda")
    x[:, 7] = torch.from_numpy(vals)
    y = call(ctx, [(m, 0, len(vals))], x, None, len(vals), n, "f32", mt.MT_ACT_NONE)
    want = vals.astype(np.float64)[:, None] * w[None, :]
    normal = np.abs(want) * 2.0 ** -24 >= 2.0 ** -126        # (so are the products of the parts of a row's value)
    assert np.array_equal(y[normal], want.astype(np.float32).astype(np.float64)[normal]) and np.all(np.abs(y - want)[~normal] <= 2.0 ** -124)
    # all 8-bit values and scales whose product with the weights 1 and -6 is an ordinary fp32 number
    q = np.array([c for c in range(256) if c & 127 != 127], dtype=np.uint8)
    x8 = np.zeros((len(q), 32), dtype=np.uint8)
    x8[:, 7] = q
    pick = [16 * 3 + 2, 16 * 3 + 15]
    for s in (10, 100, 127, 200, 240):
        y = call(ctx, [(m, 0, len(q))], torch.from_numpy(x8).cuda().view(torch.float8_e4m3fn), torch.full((len(q), 1), s, dtype=torch.uint8, device="cuda"), len(q), n,
                 "f32", mt.MT_ACT_NONE)
        assert np.array_equal(y[:, pick], lm.e4m3(q)[:, None] * 2.0 ** (s - 127) * w[pick][None, :]), s
    ctx.close()


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("rows", [5, 40, 150])
def test_infinities_and_nan_stay_in_their_rows(x_kind, rows):
    rng = np.random.default_rng(4)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, 100, 200)
    m = ctx.register_matrix4(100, 200, codes, scales)
    x, e, v = rows_in(rng, x_kind, rows, 200, 200)
    bad = [1, rows - 2]
    if x_kind == "mx8":
        x.view(torch.uint8)[1, 150] = 127
        e.view(torch.uint8)[rows - 2, 3] = 255
    else:
        x[1, 150] = float("nan")
        x[rows - 2, 20] = float("inf")
    for y_kind in ("f32", "bf16"):
        for act in (mt.MT_ACT_NONE, mt.MT_ACT_RELU, mt.MT_ACT_GELU):
            y = call(ctx, [(m, 0, rows)], x, e, rows, 100, y_kind, act)
            assert np.all(np.isnan(y[1]))
            if x_kind == "mx8":
                assert np.all(np.isnan(y[rows - 2]))
            elif act == mt.MT_ACT_NONE:
                # (0 times infinity is NaN)
                assert np.array_equal(np.isnan(y[rows - 2]), w[:, 20] == 0) and np.array_equal(y[rows - 2][w[:, 20] != 0], np.sign(w[:, 20][w[:, 20] != 0]) * np.inf)
            good = [i for i in range(rows) if i not in bad]
            check(y[good], v[good], w, None, act, x_kind, y_kind)
    ctx.close()


def test_same_answers_whatever_else_is_in_the_call():
    """A row's sums do not depend on which call it comes in, as long as the launch's shape is the same; and two calls agree bit for bit."""
    rng = np.random.default_rng(8)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, 700, 1024)
    m = ctx.register_matrix4(700, 1024, codes, scales)
    x, _, v = rows_in(rng, "bf16", 30, 1024, 1024)
    a = call(ctx, [(m, 0, 30)], x, None, 30, 700, "f32", 0)
    b = call(ctx, [(m, 0, 30)], x, None, 30, 700, "f32", 0)
    assert np.array_equal(a, b)
    ctx.close()


def test_offsets_past_32_bits():
    rng = np.random.default_rng(3)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, 40, 64)
    m = ctx.register_matrix4(40, 64, codes, scales)
    stride = (1 << 31) + 8
    buf = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 64), (stride, 1))
    x.copy_(torch.randn(3, 64))
    out = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 40), (stride, 1))
    mt.linear4(ctx, mt.row_groups([(m, 0, 3)]), x, out)
    check(out.double().cpu().numpy(), x.double().cpu().numpy(), w, None, mt.MT_ACT_NONE, "bf16", "bf16")
    ctx.close()


def test_beside_models_and_after_others_have_gone():
    """Matrices share the arena with models; a number and its place are given out again."""
    rng = np.random.default_rng(5)
    ctx = context(4 << 20)
    specs = [mt.layer_spec(mt.MT_FC, mt.MT_ACT_NONE, 64, 10)]
    small = mt.Context(2, 16, 64, 16, 4 << 20, mt.MT_F32, 0)
    wts = rng.standard_normal((10, 64)).astype(np.float32)
    small.register_model(0, specs, [wts], [None])
    kept = {}
    for i in range(12):
        n, k = int(rng.integers(1, 400)), int(rng.integers(1, 900))
        codes, scales, w = lm.random_matrix(rng, n, k)
        kept[small.register_matrix4(n, k, codes, scales)] = (n, k, w)
        if i % 3 == 2:
            gone = sorted(kept)[i % len(kept)]
            small.unregister_matrix4(gone)
            del kept[gone]
            with pytest.raises(mt.MtError) as e:
                mt.linear4(small, mt.row_groups([(gone, 0, 1)]), torch.zeros(1, 900, device="cuda"), torch.zeros(1, 400, device="cuda"))
            assert e.value.status == 3
    for m, (n, k, w) in kept.items():
        x, _, v = rows_in(rng, "f32", 4, k, k)
        check(call(small, [(m, 0, 4)], x, None, 4, n, "f32", 0), v, w, None, 0, "f32", "f32")
    x = torch.randn(3, 64, device="cuda")
    out = mt.serve(small, torch.zeros(3, dtype=torch.int32, device="cuda"), x)
    assert np.allclose(out.logits.cpu().numpy()[:, :10], x.double().cpu().numpy() @ wts.T.astype(np.float64), atol=1e-4)
    ctx.close()
    small.close()


def test_on_another_stream_and_in_a_graph():
    rng = np.random.default_rng(6)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, 500, 777)
    m = ctx.register_matrix4(500, 777, codes, scales)
    x, _, v = rows_in(rng, "bf16", 20, 777, 777)
    groups = mt.row_groups([(m, 0, 20)])
    want, y = torch.empty(20, 500, device="cuda"), torch.empty(20, 500, device="cuda")
    mt.linear4(ctx, groups, x, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mt.linear4(ctx, groups, x, y, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mt.linear4(ctx, groups, x, y)
    for i in range(3):
        x.copy_(torch.randn(20, 777))
        mt.linear4(ctx, groups, x, want)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
    ctx.close()


def test_no_rows_and_no_groups():
    rng = np.random.default_rng(7)
    ctx = context()
    codes, scales, _ = lm.random_matrix(rng, 8, 32)
    m = ctx.register_matrix4(8, 32, codes, scales)
    y = torch.full((2, 8), 7.0, device="cuda")
    x = torch.ones(2, 32, device="cuda")
    mt.linear4(ctx, mt.row_groups([]), x, y)
    mt.linear4(ctx, mt.row_groups([(m, 0, 0), (m, 2, 0)]), x, y)
    assert torch.all(y == 7.0)
    ctx.close()


def test_refusals_of_tensors():
    rng = np.random.default_rng(7)
    ctx = context()
    codes, scales, _ = lm.random_matrix(rng, 8, 64)
    m = ctx.register_matrix4(8, 64, codes, scales)
    x, y = torch.ones(4, 64, device="cuda"), torch.zeros(4, 8, device="cuda")
    one = mt.row_groups([(m, 0, 4)])
    for args, kw in (((x.half(), y), {}), ((x, y.half()), {}), ((x, y[:3]), {}), ((x.cpu(), y), {}), ((x.t().contiguous().t(), y), {}),
                     ((x, y), dict(x_scales=torch.zeros(4, 2, dtype=torch.uint8, device="cuda"))), ((x.to(torch.float8_e4m3fn), y), {})):
        with pytest.raises(ValueError):
            mt.linear4(ctx, one, *args, **kw)
    for groups, a, b, status in (([(m, 0, 5)], x, y, 1), ([(m, 4, 1)], x, y, 1), ([(m, 2, 1), (m, 1, 1)], x, y, 1), ([(m, 0, 2), (m, 1, 2)], x, y, 1), ([(m + 1, 0, 1)], x, y, 3),
                                 ([(m, 0, 4)], x[:, :63].contiguous(), y, 1), ([(m, 0, 4)], x, y[:, :7].contiguous(), 1), ([(m, 2 ** 32 - 1, 2)], x, y, 1),
                                 ([(m, 0, 1)], x[:1, :63].contiguous(), y[:1], 1)):
        with pytest.raises(mt.MtError) as e:
            mt.linear4(ctx, mt.row_groups(groups), a, b)
        assert e.value.status == status, groups
    with pytest.raises(mt.MtError) as e:
        mt.linear4(ctx, one, x, y, act=3)
    assert e.value.status == 5
    ctx.close()


def test_slices_narrower_than_their_strides_are_refused():
    """Columns of wider buffers: a matrix that needs more of them than the slice has neither reads nor writes what lies beside it."""
    rng = np.random.default_rng(7)
    ctx = context()
    codes, scales, w = lm.random_matrix(rng, 8, 64)
    m = ctx.register_matrix4(8, 64, codes, scales)
    xs, ys = torch.randn(4, 80, device="cuda"), torch.full((4, 16), 7.0, device="cuda")
    x8 = torch.zeros(4, 96, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    e8 = torch.full((4, 3), 127, dtype=torch.uint8, device="cuda")
    one = mt.row_groups([(m, 0, 4)])
    for x, y, e in ((xs[:, :63], ys[:, :8], None), (xs[:, :64], ys[:, :7], None), (xs[:, :1], ys[:, :1], None), (xs.to(torch.bfloat16)[:, :63], ys[:, :8], None),
                    (x8[:, :32], ys[:, :8], e8[:, :1]), (x8[:, :63], ys[:, :8], e8[:, :2])):
        with pytest.raises(mt.MtError) as err:
            mt.linear4(ctx, one, x, y, x_scales=e)
        assert err.value.status == 1
    torch.cuda.synchronize()
    assert torch.all(ys == 7.0)
    mt.linear4(ctx, one, xs[:, :64], ys[:, :8])
    check(ys[:, :8].double().cpu().numpy(), xs[:, :64].double().cpu().numpy(), w, None, mt.MT_ACT_NONE, "f32", "f32")
    assert torch.all(ys[:, 8:] == 7.0)
    mt.linear4(ctx, mt.row_groups([(m, 0, 4)]), xs[:, 3:67], ys[:, 8:])
    check(ys[:, 8:].double().cpu().numpy(), xs[:, 3:67].double().cpu().numpy(), w, None, mt.MT_ACT_NONE, "f32", "f32")
    ctx.close()


@pytest.mark.parametrize("y_kind", ["bf16", "f32"])
def test_gelu_of_every_size(y_kind):
    """Values themselves through a weight of 1.  z Phi(z) changes by (1 + z^2) times a relative change of z, so an error of 2^-24 in an argument of the exponential
    counts z^2 times: z^2 2^-22 and 2^-19 (bf16: 2^-16) of the result are allowed for, and its rounding."""
    from math import erfc
    ctx = context(1 << 20)
    z = np.concatenate([np.linspace(-14.0, 14.0, 3001), -np.exp2(np.linspace(-100, 3.7, 500)), np.exp2(np.linspace(-100, 100, 500)), [0.0, -0.0, -20.0, -100.0, -1e10, -1e30, 1e30]]).astype(np.float32)
    m = ctx.register_matrix4(1, 1, np.array([[2]], dtype=np.uint8), np.array([[127]], dtype=np.uint8))
    y = call(ctx, [(m, 0, len(z))], torch.from_numpy(z[:, None].copy()).cuda(), None, len(z), 1, y_kind, mt.MT_ACT_GELU)[:, 0]
    z = z.astype(np.float64)
    ref = np.array([0.5 * v * erfc(-v * 0.5 ** 0.5) for v in z])
    rel = np.minimum(z * z, 400.0) * 2.0 ** -22 + (2.0 ** -16 + 2.0 ** -8 if y_kind == "bf16" else 2.0 ** -19)
    assert np.all(np.abs(y - ref) <= rel * np.abs(ref) + (2.0 ** -133 if y_kind == "bf16" else 2.0 ** -146)), (z[np.argmax(np.abs(y - ref) - rel * np.abs(ref))])
    ctx.close()


@pytest.mark.parametrize("y_kind", ["bf16", "f32"])
def test_gelu_of_infinities_and_nan(y_kind):
    """As the definition gives it, and the layers of models: -infinity times 0 is NaN."""
    ctx = context(1 << 20)
    m = ctx.register_matrix4(1, 1, np.array([[2]], dtype=np.uint8), np.array([[127]], dtype=np.uint8))
    x = torch.tensor([[float("inf")], [-float("inf")], [float("nan")], [1.0]], device="cuda")
    y = call(ctx, [(m, 0, 4)], x, None, 4, 1, y_kind, mt.MT_ACT_GELU)[:, 0]
    assert y[0] == np.inf and np.isnan(y[1]) and np.isnan(y[2]) and abs(y[3] - 0.8413447) < 2.0 ** -8
    ctx.close()


@pytest.mark.parametrize("n,k", [(64, 32), (4096, 1056)])
def test_8_bit_rows_of_every_scale(n, k):
    """Every value at every scale, against weights that bring the product back into fp32's range: exact from 2^-124 to 2^119 (bytes 3 .. 246); at smaller scales bits
    below 2^-133 are lost, at larger ones what bf16 cannot hold is infinite."""
    ctx = context()
    q = np.array([c for c in range(256) if c & 127 != 127], dtype=np.uint8)
    x8 = np.zeros((len(q), k), dtype=np.uint8)
    x8[:, 7] = q
    for weight_scale, bytes_ in ((227, (0, 1, 2, 3, 4, 9)), (127, (60, 127, 190)), (27, (230, 241, 245, 246, 247, 248, 254))):
        codes = np.zeros((n, k // 2), dtype=np.uint8)
        codes[:, 3] = (np.arange(n) % 2 * 8 + 2) << 4                 # column 7: 1 and -1
        m = ctx.register_matrix4(n, k, codes, np.full((n, k // 32), weight_scale, dtype=np.uint8))
        sign = np.where(np.arange(n) % 2, -1.0, 1.0)
        for s in bytes_:
            scales = np.full((len(q), k // 32), 127, dtype=np.uint8)
            scales[:, 0] = s
            y = call(ctx, [(m, 0, len(q))], torch.from_numpy(x8).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda(), len(q), n, "f32", mt.MT_ACT_NONE)
            v = lm.e4m3(q) * 2.0 ** (s - 127.0)
            want = v[:, None] * sign[None, :] * 2.0 ** (weight_scale - 127.0)
            if s < 3:
                assert np.all(np.abs(y - want) <= 2.0 ** -133 * 2.0 ** (weight_scale - 127.0)), s
            elif s < 247:
                assert np.array_equal(y, want), s
            else:
                fits = np.abs(v) <= (2 - 2.0 ** -7) * 2.0 ** 127
                assert np.array_equal(y[fits], want[fits]) and np.array_equal(y[~fits], np.sign(want[~fits]) * np.inf), s
        ctx.unregister_matrix4(m)
    ctx.close()


# ---- rows through LDS -----------------------------------------------------------------------------
KIND = {"f32": mt.MT_F32, "bf16": mt.MT_BF16, "mx8": mt.MT_MX8}
# (rows, out_features, in_features) of every tenant: ends of outputs of every kind, workgroups' outputs that are no multiple of eight, fan-ins of less than a vector, than a tile,
# than a round of four, whole and not; in the second set also rows in several chunks
LDS_SETS = {
    "few rows": [(24, 2064, 1100), (32, 2061, 1152), (17, 2100, 1024), (31, 2070, 1537), (0, 50, 300), (32, 2048, 1030), (1, 2077, 100), (30, 2064, 5), (29, 2063, 640), (25, 2050, 1283), (20, 130, 127), (32, 2300, 1),
                 (26, 2064, 1025)],
    "many rows": [(64, 2600, 1100), (50, 2609, 1152), (150, 2603, 1029), (64, 2563, 100), (63, 2600, 5), (1, 2600, 1536), (49, 2690, 1024), (60, 2561, 1283), (2, 17, 300), (64, 2600, 1)],
}


def lds_form(groups, x_kind):
    """That the call takes rows through LDS, and the rows of a workgroup."""
    s = mt.debug_linear4_shape(groups, torch.cuda.get_device_properties(0).multi_processor_count, KIND[x_kind])
    assert s["through_lds"] and s["outputs"] == 128, s
    return s["rows"]


@pytest.fixture(scope="module", params=list(LDS_SETS))
def lds_set(request):
    """(groups' sizes, context, numbers, (weights, biases), first rows, rows) of a set; every other matrix has biases."""
    rng = np.random.default_rng(len(request.param))
    ctx = context(128 << 20)
    numbers, values, first, at = [], [], [], 3
    for i, (rows, n, k) in enumerate(LDS_SETS[request.param]):
        codes, scales, w = lm.random_matrix(rng, n, k)
        bias = rng.standard_normal(n).astype(np.float32) if i % 2 == 0 else None
        numbers.append(ctx.register_matrix4(n, k, codes, scales, bias))
        values.append((w, bias))
        first.append(at)
        at += rows + i % 2                       # (every other group is followed by a row of nobody)
    yield LDS_SETS[request.param], ctx, numbers, values, first, at
    ctx.close()


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("y_kind", ["bf16", "f32"])
@pytest.mark.parametrize("act", [mt.MT_ACT_NONE, mt.MT_ACT_RELU, mt.MT_ACT_GELU])
def test_groups_whose_rows_go_through_lds(lds_set, x_kind, y_kind, act):
    sizes, ctx, numbers, values, first, total = lds_set
    rng = np.random.default_rng(act)
    assert lds_form(sizes, x_kind) == (16 if x_kind == "f32" else 32 if max(r for r, _, _ in sizes) <= 32 else 64)
    x, e, v = rows_in(rng, x_kind, total, 1537, 1537 + 3 * act, act)
    stride = 2700
    buf = torch.full((total * stride + 8,), 7.0, dtype=DT[y_kind], device="cuda")
    y = buf[:total * stride].view(total, stride)
    mt.linear4(ctx, mt.row_groups(zip(numbers, first, [s[0] for s in sizes])), x, y[:, :2690], x_scales=e, act=act)
    y = y.double().cpu().numpy()
    of_somebody = np.zeros(total, dtype=bool)
    for (rows, n, k), (w, bias), at in zip(sizes, values, first):
        assert np.all(y[at:at + rows, n:] == 7.0)
        of_somebody[at:at + rows] = True
        some = at + np.unique(np.concatenate([[0, rows - 1, rows // 2], rng.integers(0, rows, 5)])) if rows else []
        if rows:
            check(y[some, :n], v[some, :k], w, bias, act, x_kind, y_kind)
    assert np.all(y[~of_somebody] == 7.0) and bool((buf[total * stride:] == 7.0).all())


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
def test_rows_through_lds_whatever_else_is_in_the_call(lds_set, x_kind):
    """A row's sums are the same bits with and without other groups, as long as rows go through LDS."""
    sizes, ctx, numbers, _, first, total = lds_set
    x, e, _ = rows_in(np.random.default_rng(1), x_kind, total, 1537, 1540)
    whole = torch.zeros(total, 2690, device="cuda")
    groups = list(zip(numbers, first, [s[0] for s in sizes]))
    mt.linear4(ctx, mt.row_groups(groups), x, whole, x_scales=e)
    tried = 0
    for left_out in ([1], [0, 4], [2, 7, 8]):
        kept = [i for i in range(len(sizes)) if i not in left_out]
        try:
            lds_form([sizes[i] for i in kept], x_kind)
        except AssertionError:
            continue
        tried += 1
        some = torch.zeros_like(whole)
        mt.linear4(ctx, mt.row_groups([groups[i] for i in kept]), x, some, x_scales=e)
        for i, (m, at, rows) in enumerate(groups):
            assert torch.equal(some[at:at + rows], whole[at:at + rows] if i in kept else torch.zeros_like(whole[at:at + rows])), (left_out, i)
    assert tried


@pytest.mark.parametrize("x_kind", ["bf16", "f32", "mx8"])
@pytest.mark.parametrize("y_kind", ["bf16", "f32"])
def test_infinities_and_nan_through_lds(lds_set, x_kind, y_kind):
    """They stay in their rows, beside numbers of every size in the same vectors; in whole tiles of the fan-in and in the last."""
    sizes, ctx, numbers, values, first, total = lds_set
    lds_form(sizes, x_kind)
    groups = mt.row_groups(zip(numbers, first, [s[0] for s in sizes]))
    x, e, v = rows_in(np.random.default_rng(2), x_kind, total, 1537, 1537)
    rows, n, k = sizes[0]                        # (k = 1100: its last tile is not whole)
    (w, bias), at = values[0], first[0]
    bad = {}
    for i, col in enumerate((7, 511, 1023, 1024, 1090, k - 1)):
        if x_kind == "mx8":
            x.view(torch.uint8)[at + 2 * i, col] = 127
            e.view(torch.uint8)[at + 2 * i + 1, col // 32] = 255
            bad[at + 2 * i] = bad[at + 2 * i + 1] = None
        else:
            what = (float("inf"), -float("inf"))[i % 2]
            x[at + 2 * i, col] = float("nan")
            x[at + 2 * i + 1, col] = what
            bad[at + 2 * i], bad[at + 2 * i + 1] = None, (col, what)
            x[at + 2 * i + 1, col - 1] = 3.0e38 if i % 2 else 1.0e-38        # (beside an infinity neither counts)
    for act in (mt.MT_ACT_NONE, mt.MT_ACT_RELU, mt.MT_ACT_GELU):
        y = torch.zeros(total, 2690, dtype=DT[y_kind], device="cuda")
        mt.linear4(ctx, groups, x, y, x_scales=e, act=act)
        y = y.double().cpu().numpy()
        for r, why in bad.items():
            if why is None:
                assert np.all(np.isnan(y[r, :n])), (act, r)
                continue
            with np.errstate(invalid="ignore"):
                z = w[:, why[0]] * why[1]        # (0 times infinity is NaN)
                want = {mt.MT_ACT_NONE: z, mt.MT_ACT_RELU: np.where(z < 0, 0.0, z), mt.MT_ACT_GELU: np.where(z == -np.inf, np.nan, z)}[act]
            assert np.array_equal(y[r, :n], want, equal_nan=True), (act, r)
        for (rows_g, n_g, k_g), (w_g, b_g), at_g in zip(sizes, values, first):
            good = [r for r in range(at_g, at_g + rows_g) if r not in bad][:6]
            if good:
                check(y[good, :n_g], v[good, :k_g], w_g, b_g, act, x_kind, y_kind)
