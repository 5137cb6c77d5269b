"""mt_add_norm against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import lm_common as lm
import paper_1901_06887_amd as mt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# A row's squares are summed by at least 64 lanes in runs, then in trees: at most 60 additions behind one another for the widths here, half of their
# relative error in the root; six more roundings up to y.  (60 / 2 + 6) * 2^-24 = 2.2e-6.
REL = 3e-6
HALF_ULP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx():
    c = mt.Context(1, 1, 64, 1, 1 << 16, mt.MT_BF16, 0)
    yield c
    c.close()


def rows_in(rng, rows, width, stride, dtype, offset=0, fill=float("nan"), scale=1.0):
    """(view, values) of rows at odd places of a buffer full of NaN."""
    buf = torch.full((offset + rows * stride + 8,), fill, dtype=DT[dtype])
    v = buf[offset:offset + rows * stride].view(rows, stride)[:, :width]
    v.copy_(torch.from_numpy(rng.standard_normal((rows, width)) * scale))
    buf = buf.cuda()
    return buf[offset:offset + rows * stride].view(rows, stride)[:, :width], v.double().numpy()


def bytes_in(rows, width, stride, dtype):
    buf = torch.full((rows * stride + 8,), 0xa5, dtype=torch.uint8, device="cuda")
    return buf, buf[:rows * stride].view(rows, stride)[:, :width].view(dtype)


def check(h, gain, eps, dtype, y=None, q=None, scales=None):
    """y, q, scales (numpy: float64, bytes, bytes) against rows h of exact sums."""
    ref = h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * gain
    if y is not None:
        assert np.all(np.abs(y - ref) <= (HALF_ULP[dtype] + REL) * np.abs(ref) + 1e-38), np.max(np.abs(y - ref) / np.maximum(np.abs(ref), 1e-30))
    if q is not None:
        width = h.shape[1]
        pad = np.zeros((h.shape[0], -width % 32))
        most = np.abs(np.concatenate([ref, pad], 1)).reshape(h.shape[0], -1, 32).max(2)
        s = lm.e8m0(scales)
        assert np.all(s[most == 0] == 1)
        at = most > 448 * 2.0 ** -126
        assert np.all(most[at] <= 448 * s[at] * (1 + REL)) and np.all(most[at] > 224 * s[at] * (1 - REL))
        assert np.all(s[(most > 0) & ~at] == 2.0 ** -126)
        step = lm.spread(s, width)
        assert np.all(np.abs(lm.e4m3(q) * step - ref) <= np.maximum(2.0 ** -4 * np.abs(ref), 2.0 ** -10 * step) * (1 + 1e-5) + REL * np.abs(ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 7, 31, 32, 33, 100, 511, 512, 513, 1000, 1024, 1025, 1531, 2048, 2049, 4096, 4100, 8192, 8200, 16384, 16392, 40001])
def test_rows_of_any_width(ctx, dtype, width):
    rng = np.random.default_rng(width)
    rows = 5
    x, xv = rows_in(rng, rows, width, width + 3, dtype, 1)
    r, rv = rows_in(rng, rows, width, width + 1, dtype, 3, scale=0.3)
    gain, gv = rows_in(rng, 1, width, width + 5, "f32", 1)
    buf_s = torch.full((rows * (width + 2) + 8,), 7.0, dtype=DT[dtype], device="cuda")
    buf_y = torch.full((rows * (width + 9) + 8,), 7.0, dtype=DT[dtype], device="cuda")
    s, y = buf_s[:rows * (width + 2)].view(rows, -1)[:, :width], buf_y[:rows * (width + 9)].view(rows, -1)[:, :width]
    n = -(-width // 32)
    buf_q, q = bytes_in(rows, width, width + 7, torch.float8_e4m3fn)
    buf_e, e = bytes_in(rows, n, n + 1, torch.float8_e8m0fnu)
    mt.add_norm(ctx, x, r, gain, eps=1e-5, sum_out=s, out=y, out8=q, out8_scales=e)
    torch.cuda.synchronize()
    assert torch.equal(s, (x.float() + r.float()).to(DT[dtype]))
    check(xv + rv, gv, 1e-5, dtype, y.double().cpu().numpy(), q.view(torch.uint8).cpu().numpy(), e.view(torch.uint8).cpu().numpy())
    # nothing between and behind the rows is written
    for buf, stride, wide in ((buf_s, width + 2, width), (buf_y, width + 9, width)):
        assert torch.all(buf[:rows * stride].view(rows, -1)[:, wide:] == 7.0) and torch.all(buf[rows * stride:] == 7.0)
    for buf, stride, wide in ((buf_q, width + 7, width), (buf_e, n + 1, n)):
        assert torch.all(buf[:rows * stride].view(rows, -1)[:, wide:] == 0xa5) and torch.all(buf[rows * stride:] == 0xa5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width", [(1, 1024), (2, 64), (777, 300), (4097, 96), (130, 6000)])
def test_many_rows_and_every_set_of_outputs(ctx, dtype, rows, width):
    rng = np.random.default_rng(rows)
    x, xv = rows_in(rng, rows, width, width, dtype)
    r, rv = rows_in(rng, rows, width, width, dtype)
    gain, gv = rows_in(rng, 3, width, width, "f32")
    ids = torch.from_numpy(rng.integers(0, 3, rows).astype(np.int32)).cuda()
    for residual, with_gain, s, y, q in ((1, 1, 1, 1, 1), (1, 0, 1, 0, 0), (0, 1, 0, 1, 0), (0, 2, 0, 0, 1), (1, 2, 0, 1, 1), (0, 0, 1, 1, 0)):
        sum_out, out = torch.zeros_like(x) if s else None, torch.zeros_like(x) if y else None
        out8 = torch.zeros(rows, width, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) if q else None
        scales = torch.zeros(rows, -(-width // 32), dtype=torch.uint8, device="cuda") if q else None
        mt.add_norm(ctx, x, r if residual else None, (None, gain[:1], gain)[with_gain], ids if with_gain == 2 else None, sum_out=sum_out, out=out, out8=out8,
                    out8_scales=scales)
        h = xv + rv if residual else xv
        g = (1.0, gv[:1], gv[ids.cpu().numpy()])[with_gain]
        check(h, g, 1e-6, dtype, out.double().cpu().numpy() if y else None, out8.view(torch.uint8).cpu().numpy() if q else None, scales.cpu().numpy() if q else None)
        if s:
            assert torch.equal(sum_out, ((x.float() + r.float()) if residual else x.float()).to(DT[dtype]))


@pytest.mark.parametrize("width", [40, 1024, 4096, 20000])
def test_outputs_in_place(ctx, width):
    rng = np.random.default_rng(9)
    x, xv = rows_in(rng, 6, width, width, "bf16")
    r, rv = rows_in(rng, 6, width, width, "bf16")
    h = (x.float() + r.float()).to(torch.bfloat16)
    for place in ("x", "residual"):
        a, b = x.clone(), r.clone()
        y = torch.empty_like(x)
        mt.add_norm(ctx, a, b, sum_out=a if place == "x" else b, out=y)
        assert torch.equal(a if place == "x" else b, h) and torch.equal(b if place == "x" else a, r if place == "x" else x)
        check(xv + rv, 1.0, 1e-6, "bf16", y.double().cpu().numpy())
        a, b = x.clone(), r.clone()
        mt.add_norm(ctx, a, b, out=a if place == "x" else b)
        check(xv + rv, 1.0, 1e-6, "bf16", (a if place == "x" else b).double().cpu().numpy())


def test_rows_of_unknown_tenants_touch_no_gain(ctx):
    rng = np.random.default_rng(2)
    x, xv = rows_in(rng, 6, 100, 100, "f32")
    gain, gv = rows_in(rng, 2, 100, 100, "f32")
    ids = torch.tensor([0, 1, 2, -1, 2 ** 31 - 1, 1], dtype=torch.int32, device="cuda")
    s, y = torch.full_like(x, 7), torch.full_like(x, 7)
    q, e = torch.full((6, 100), 7, dtype=torch.uint8, device="cuda"), torch.full((6, 4), 7, dtype=torch.uint8, device="cuda")
    mt.add_norm(ctx, x, None, gain, ids, sum_out=s, out=y, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    assert torch.equal(s, x)
    known, unknown = [0, 1, 5], [2, 3, 4]
    assert torch.all(y[unknown] == 0) and torch.all(q[unknown] == 0) and torch.all(e[unknown] == 127)
    check(xv[known], gv[[0, 1, 1]], 1e-6, "f32", y[known].double().cpu().numpy(), q[known].cpu().numpy(), e[known].cpu().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_infinities_and_nan(ctx, dtype):
    x = torch.ones(5, 96, dtype=DT[dtype], device="cuda")
    x[0] = 0                                    # a row of zeros
    x[1, 40] = float("nan")
    x[2, 40] = float("inf")
    x[3, 32:64] = 0                             # a block of zeros
    y, q, e = torch.empty_like(x), torch.empty(5, 96, dtype=torch.uint8, device="cuda"), torch.empty(5, 3, dtype=torch.uint8, device="cuda")
    mt.add_norm(ctx, x, out=y, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    assert torch.all(y[0] == 0) and torch.all(q[0] == 0) and torch.all(e[0] == 127)
    assert torch.all(torch.isnan(y[1])) and torch.all(e[1] == 255) and torch.all(q[1] == 127)
    # the infinity divided by itself is NaN, everything else of its row 0
    assert torch.isnan(y[2, 40]) and int((y[2] == 0).sum()) == 95
    assert e[2].tolist() == [127, 255, 127] and torch.all(q[2, 32:64] == 127) and torch.all(q[2, :32] == 0)
    check(x[3:].double().cpu().numpy(), 1.0, 1e-6, dtype, y[3:].double().cpu().numpy(), q[3:].cpu().numpy(), e[3:].cpu().numpy())
    assert e[3, 1] == 127 and torch.all(q[3, 32:64] == 0)


def test_an_infinite_gain_spoils_its_block_alone(ctx):
    x = torch.ones(1, 100, device="cuda")
    gain = torch.ones(100, device="cuda")
    gain[70] = float("inf")
    q, e = torch.empty(1, 100, dtype=torch.uint8, device="cuda"), torch.empty(1, 4, dtype=torch.uint8, device="cuda")
    mt.add_norm(ctx, x, gain=gain, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    assert e[0, 2] == 255 and torch.all(q[0, 64:96] == 127) and int((e == 255).sum()) == 1 and not torch.any(q[0, :64] == 127) and not torch.any(q[0, 96:] == 127)


def test_scales_reach_from_the_smallest_to_the_largest(ctx):
    """Blocks of one magnitude each, and magnitudes on both sides of 448 times a power of two."""
    gain = torch.tensor([2.0 ** -126, 2.0 ** -119, 448.0 * 2.0 ** -126, 2.0 ** -100, 1.0, 448.0, 448.0 * (1 + 2.0 ** -20), 500.0, 2.0 ** 100, 2.0 ** 127], device="cuda")
    x = torch.ones(1, 320, device="cuda")
    q, e = torch.empty(1, 320, dtype=torch.uint8, device="cuda"), torch.empty(1, 10, dtype=torch.uint8, device="cuda")
    mt.add_norm(ctx, x, gain=gain.repeat_interleave(32), eps=0.0, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    assert (e[0].cpu().numpy().astype(int) - 127).tolist() == [-126, -126, -126, -108, -8, 0, 1, 1, 92, 119]
    v = lm.e4m3(q.cpu().numpy()) * lm.spread(lm.e8m0(e.cpu().numpy()), 320)
    want = gain.repeat_interleave(32).double().cpu().numpy()
    assert np.all(np.abs(v[0] - want) <= np.maximum(2.0 ** -4 * want, 2.0 ** -10 * 2.0 ** -126))


def test_offsets_past_32_bits(ctx):
    rows, stride = 3, (1 << 31) + 5
    buf = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, 64), (stride, 1))
    x.copy_(torch.randn(rows, 64))
    y = torch.empty(rows, 64, dtype=torch.bfloat16, device="cuda")
    mt.add_norm(ctx, x, out=y)
    check(x.double().cpu().numpy(), 1.0, 1e-6, "bf16", y.double().cpu().numpy())


def test_more_rows_than_a_grid_of_threads(ctx):
    rows, width = (2 << 21) + 3, 4
    x, r = torch.randn(rows, width, device="cuda"), torch.randn(rows, width, device="cuda")
    gain, ids = torch.randn(5, width, device="cuda"), torch.randint(-1, 6, (rows,), dtype=torch.int32, device="cuda")
    s, y = torch.empty_like(x), torch.empty_like(x)
    q, e = torch.empty(rows, width, dtype=torch.uint8, device="cuda"), torch.empty(rows, 1, dtype=torch.uint8, device="cuda")
    mt.add_norm(ctx, x, residual=r, gain=gain, gain_ids=ids, sum_out=s, out=y, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    h = x + r
    assert torch.equal(s, h)
    known = (ids >= 0) & (ids < 5)
    g = gain.double()[ids.clamp(0, 4).long()] * known.double()[:, None]
    want = h.double() * torch.rsqrt((h.double() ** 2).mean(1, keepdim=True) + 1e-6) * g
    assert bool(((y.double() - want).abs() <= (REL + HALF_ULP["f32"]) * want.abs() + 1e-38).all())
    for first in (0, (1 << 21) - 5, (2 << 21) - 5, rows - 8):                    # the 8-bit rows are those of calls of a few rows
        few = slice(first, first + 8)
        q1, e1 = torch.empty(8, width, dtype=torch.uint8, device="cuda"), torch.empty(8, 1, dtype=torch.uint8, device="cuda")
        mt.add_norm(ctx, x[few], residual=r[few], gain=gain, gain_ids=ids[few], out8=q1.view(torch.float8_e4m3fn), out8_scales=e1)
        assert torch.equal(q[few], q1) and torch.equal(e[few], e1)


def test_on_another_stream_and_in_a_graph(ctx):
    x = torch.randn(40, 4096, dtype=torch.bfloat16, device="cuda")
    want, y = torch.empty_like(x), torch.empty_like(x)
    mt.add_norm(ctx, x, out=want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    mt.add_norm(ctx, x, out=y, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mt.add_norm(ctx, x, out=y)
    for k in range(3):
        x.copy_(torch.randn(40, 4096).to(torch.bfloat16))
        mt.add_norm(ctx, x, out=want)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), k


def test_no_rows(ctx):
    x = torch.empty(0, 64, device="cuda")
    mt.add_norm(ctx, x, out=torch.empty_like(x))


def test_refusals_of_tensors(ctx):
    x = torch.ones(4, 64, device="cuda")
    bad = [dict(out=torch.empty(4, 63, device="cuda")), dict(out=torch.empty(4, 64, dtype=torch.bfloat16, device="cuda")), dict(out=torch.empty(4, 64)),
           dict(out=torch.empty(64, 4, device="cuda").t()), dict(out=x, residual=torch.ones(3, 64, device="cuda")), dict(out=x, gain=torch.ones(63, device="cuda")),
           dict(out=x, gain=torch.ones(2, 64, device="cuda"), gain_ids=torch.zeros(4, dtype=torch.int64, device="cuda"))]
    for kw in bad:
        with pytest.raises(ValueError):
            mt.add_norm(ctx, x, **kw)
    for kw in (dict(), dict(out=x.clone(), eps=-1.0), dict(out=x.clone(), eps=float("nan")), dict(out8=torch.empty(4, 64, dtype=torch.float8_e4m3fn, device="cuda"))):
        with pytest.raises(mt.MtError) as e:
            mt.add_norm(ctx, x, **kw)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        mt.add_norm(ctx, x.half(), out=x.half())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 40, 500, 1000, 4096, 9000, 20000])
@pytest.mark.parametrize("eps", [0.0, 1e-35, 1e-6, 1e30])
def test_rows_whose_squares_leave_the_range(ctx, dtype, width, eps):
    """Finite rows of any magnitude: their squares' sum may lie beyond fp32's largest number, or below its smallest."""
    rng = np.random.default_rng(width)
    sizes = np.array([1.0, 1e20, 1e38, 3e18, 1e-18, 1e-25, 1e-37, 1e-39, 1.0])
    rows = len(sizes)
    v = rng.uniform(0.3, 3.0, (rows, width)) * rng.choice([-1.0, 1.0], (rows, width)) * sizes[:, None]
    v[8, ::2] *= 1e36
    v[8, 1::2] *= 1e-36
    x = torch.from_numpy(v).to(DT[dtype]).cuda()
    xv = x.double().cpu().numpy()
    gain, gv = rows_in(rng, 1, width, width, "f32")
    for residual in (False, True):
        a = (x.double() * 0.75).to(DT[dtype]) if residual else x
        r = (x.double() - a.double()).to(DT[dtype]) if residual else None
        h = a.double().cpu().numpy() + (r.double().cpu().numpy() if residual else 0.0)
        h = h.astype(np.float32).astype(np.float64)
        s, y = torch.empty_like(x) if residual else None, torch.empty_like(x)
        q, e = torch.empty(rows, width, dtype=torch.uint8, device="cuda"), torch.empty(rows, -(-width // 32), dtype=torch.uint8, device="cuda")
        mt.add_norm(ctx, a, r, gain, eps=eps, sum_out=s, out=y, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
        if residual:
            assert torch.equal(s.double().cpu(), torch.from_numpy(h).to(DT[dtype]).double())
        yv, qv, ev = y.double().cpu().numpy(), q.cpu().numpy(), e.cpu().numpy()
        check(h, gv, float(np.float32(eps)), dtype, yv)
        # rows whose every value is below fp32's smallest are zeros, and zeros have the scale 1
        gone = np.abs(h / np.sqrt((h * h).mean(1, keepdims=True) + float(np.float32(eps))) * gv).max(1) < 2.0 ** -150
        check(h[~gone], gv, float(np.float32(eps)), dtype, yv[~gone], qv[~gone], ev[~gone])
        assert np.all(yv[gone] == 0) and np.all(qv[gone] & 127 == 0) and np.all(ev[gone] == 127)


def test_zero_rows_and_infinities_without_eps(ctx):
    """0 / 0 is NaN; an infinity's row stays as with an eps."""
    x = torch.zeros(3, 600, device="cuda")
    x[1] = 1e30
    x[1, 7] = float("inf")
    x[2, 3] = 1e-44
    y = torch.empty_like(x)
    mt.add_norm(ctx, x, eps=0.0, out=y)
    assert torch.all(torch.isnan(y[0])) and torch.isnan(y[1, 7]) and int((y[1] == 0).sum()) == 599
    assert int((y[2] == 0).sum()) == 599 and abs(float(y[2, 3]) - 600 ** 0.5) < 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,width,pad", [(15000, 512, 0), (15000, 505, 3), (3000, 4100, 1), (4400, 2048, 8), (1100, 10000, 5), (700, 20000, 0), (700, 20011, 2)])
@pytest.mark.parametrize("place", [None, "x", "residual"])
def test_outputs_larger_than_the_caches(ctx, dtype, rows, width, pad, place):
    """Above 32 MiB of outputs these go past the caches: wide and cut-off runs, rows that are read twice, sums in place."""
    assert rows * width * 5 > 32 << 20
    rng = np.random.default_rng(width)
    g = torch.Generator("cuda").manual_seed(width)
    wide = lambda t, p, fill: torch.full((rows * (width + p) + 8,), fill, dtype=t, device="cuda")  # noqa: E731
    rows_of = lambda buf, p: buf[:rows * (width + p)].view(rows, -1)[:, :width]  # noqa: E731
    buf_x, buf_r, buf_y, buf_q = wide(DT[dtype], pad, 7.0), wide(DT[dtype], pad, 7.0), wide(DT[dtype], 2 * pad, 7.0), wide(torch.uint8, pad, 0xa5)
    x, r, y, q = rows_of(buf_x, pad), rows_of(buf_r, pad), rows_of(buf_y, 2 * pad), rows_of(buf_q, pad)
    x.copy_(torch.randn(rows, width, generator=g, device="cuda"))
    r.copy_(torch.randn(rows, width, generator=g, device="cuda") * 0.3)
    gain, gv = rows_in(rng, 4, width, width, "f32")
    ids = torch.from_numpy(rng.integers(0, 4, rows).astype(np.int32)).cuda()
    n = -(-width // 32)
    e = torch.full((rows, n), 0xa5, dtype=torch.uint8, device="cuda")
    h32 = x.float() + r.float()
    h = x.double() + r.double()
    kept = {"x": r.clone(), "residual": x.clone()}.get(place)
    s = {None: torch.full_like(x, 7.0), "x": x, "residual": r}[place]
    mt.add_norm(ctx, x, r, gain, ids, eps=1e-5, sum_out=s, out=y, out8=q.view(torch.float8_e4m3fn), out8_scales=e)
    assert torch.equal(s, h32.to(DT[dtype]))
    if kept is not None:
        assert torch.equal(r if place == "x" else x, kept)
    ref = h * torch.rsqrt((h * h).mean(1, keepdim=True) + float(np.float32(1e-5))) * gain.double()[ids.long()]
    assert bool(((y.double() - ref).abs() <= (HALF_ULP[dtype] + REL) * ref.abs() + 1e-38).all())
    for buf, p, fill in ((buf_x, pad, 7.0), (buf_r, pad, 7.0), (buf_y, 2 * pad, 7.0), (buf_q, pad, 0xa5)):
        assert bool((buf[:rows * (width + p)].view(rows, -1)[:, width:] == fill).all()) and bool((buf[rows * (width + p):] == fill).all())
    some = np.unique(np.concatenate([[0, 1, rows - 2, rows - 1], rng.integers(0, rows, 60)]))
    at = torch.from_numpy(some).cuda()
    check(h[at].cpu().numpy(), gv[ids[at].cpu().numpy()], 1e-5, dtype, None, q[at].cpu().numpy(), e[at].cpu().numpy())
    # and the 8-bit rows are those of calls of a few rows
    for first in (0, rows // 2, rows - 9):
        few = slice(first, first + 9)
        q1, e1 = torch.empty(9, width, dtype=torch.uint8, device="cuda"), torch.empty(9, n, dtype=torch.uint8, device="cuda")
        if place is None:
            mt.add_norm(ctx, x[few], r[few], gain, ids[few], eps=1e-5, out8=q1.view(torch.float8_e4m3fn), out8_scales=e1)
            assert torch.equal(q[few], q1) and torch.equal(e[few], e1)
