"""mt_score against softmax, entropy and order in 64 bits."""
import numpy as np
import pytest
import torch

import lm_common as lm
import paper_1901_06887_amd as mt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
LOWEST = {"bf16": -3.3895313892515355e38, "f32": -3.4028234663852886e38}


@pytest.fixture(scope="module")
def ctx():
    c = mt.Context(1, 1, 64, 1, 1 << 16, mt.MT_BF16, 0)
    yield c
    c.close()


def agree(o, ref, n_given, top):
    """Whole numbers equal, infinities and NaN in the same places, the rest within what fp32 explains."""
    def near(a, b, bound):
        with np.errstate(over="ignore"):
            a, b = a.double().cpu().numpy(), np.asarray(b).astype(np.float32).astype(np.float64)      # (beyond fp32's range: an infinity)
        assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(np.isneginf(a), np.isneginf(b))
        fine = np.isfinite(b)
        off = np.where(fine, np.abs(np.where(fine, a, 0) - np.where(fine, b, 0)), 0)
        assert np.all(off <= bound + 2.0 ** -21 * np.abs(np.where(fine, b, 0))), (off.max(), np.unravel_index(np.argmax(off), off.shape))

    near(o.entropy, ref["entropy"], ref["bound"])
    if n_given:
        assert np.array_equal(o.given_ranks.cpu().numpy(), ref["ranks"])
        near(o.given_logprobs, ref["given"], ref["bound"][:, None])
    if top:
        assert np.array_equal(o.top_ids.cpu().numpy(), ref["ids"])
        near(o.top_logprobs, ref["top"], ref["bound"][:, None])


def dev_bits(allowed):
    return None if allowed is None else torch.from_numpy(allowed.view(np.int32)).cuda()


def run(ctx, x, given=None, n=None, allowed=None, top=0, temperature=1.0, out=None):
    """The call on device logits x, and the reference on the same values."""
    o = out or mt.alloc_scores(x.shape[0], 0 if given is None else given.shape[1], top)
    for t in (o.given_logprobs, o.given_ranks, o.entropy, o.top_ids, o.top_logprobs):
        if t is not None:
            t.fill_(77)
    mt.score(ctx, x, o, given=None if given is None else torch.from_numpy(given.astype(np.int32)).cuda(), n_classes=None if n is None else torch.from_numpy(n.astype(np.int32)).cuda(),
             allowed=dev_bits(allowed), temperature=temperature)
    torch.cuda.synchronize()
    ref = lm.scored(x.double().cpu().numpy(), n, allowed, given, top, float(np.float32(temperature)))
    agree(o, ref, 0 if given is None else given.shape[1], top)
    return o


def logits(rng, rows, classes, dtype, stride=None, offset=0, scale=3.0):
    stride = stride or classes
    buf = torch.full((offset + rows * stride + 16,), float("nan"), dtype=DT[dtype], device="cuda")
    v = buf[offset:offset + rows * stride].view(rows, stride)[:, :classes]
    v.copy_(torch.from_numpy(rng.standard_normal((rows, classes)) * scale))
    return v


def bits(rng, rows, classes, share):
    ok = rng.random((rows, -(-classes // 32) * 32)) < share
    return np.packbits(ok, axis=1, bitorder="little").view(np.uint32).copy()


CLASSES = [1, 2, 3, 10, 31, 63, 64, 65, 255, 256, 257, 1000, 1023, 1024, 2047, 2048, 2049, 4097, 10007, 32768, 65001, 131072]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", CLASSES)
def test_numbers_of_classes(ctx, dtype, classes):
    rng = np.random.default_rng(classes)
    for i, (rows, n_given, top) in enumerate(((1, 1, 5), (3, 16, 32), (2, 0, 1), (5, 3, 0))):
        x = logits(rng, rows, classes, dtype, classes + (0, 1, 3, 64)[i], i)
        given = rng.integers(0, classes, (rows, n_given)) if n_given else None
        run(ctx, x, given, top=top, temperature=(1.0, 0.7, 3.0, 1.0)[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [5, 100, 1000, 5000, 70001])
def test_masks_and_class_counts(ctx, dtype, classes):
    rng = np.random.default_rng(classes + 1)
    rows = 9
    x = logits(rng, rows, classes, dtype, classes + 1, 1)
    given = rng.integers(-2, classes + 2, (rows, 4))
    n = rng.integers(0, classes + 1, rows)
    n[0], n[1], n[2], n[3] = 0, -5, classes + 9, 1
    for share in (0.0, 0.003, 0.5, 1.0):
        m = bits(rng, rows, classes, share)
        m[4] = 0                                 # nothing allowed
        m[5, :] = 0
        m[5, (classes - 1) // 32] = 1 << ((classes - 1) % 32)        # only the last class
        run(ctx, x, given, None, m, 20)
        run(ctx, x, given, n, m, 20)
    run(ctx, x, given, n, None, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [40, 700, 3001, 65001])
def test_what_stands_in_masked_places_does_not_matter(ctx, dtype, classes):
    rng = np.random.default_rng(classes + 2)
    x = logits(rng, 6, classes, dtype)
    m = bits(rng, 6, classes, 0.5)
    off = torch.from_numpy(np.unpackbits(m.view(np.uint8), axis=1, bitorder="little")[:, :classes] == 0).cuda()
    want = run(ctx, x, rng.integers(0, classes, (6, 2)), None, m, 10)
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"), LOWEST[dtype], -LOWEST[dtype])):
        y = torch.where(off, torch.tensor(v, dtype=DT[dtype], device="cuda"), x)
        o = run(ctx, y, rng.integers(0, classes, (6, 2)), None, m, 10)
        assert torch.equal(o.entropy, want.entropy) and torch.equal(o.top_ids, want.top_ids) and torch.equal(o.top_logprobs, want.top_logprobs)
    # the same classes taken out by -infinity, or by the class count, where NaN follows
    o = run(ctx, torch.where(off, torch.tensor(-float("inf"), dtype=DT[dtype], device="cuda"), x), rng.integers(0, classes, (6, 2)), top=10)
    assert torch.equal(o.top_ids, want.top_ids)
    y = x.clone()
    n = rng.integers(1, classes, 6)
    for r in range(6):
        y[r, n[r]:] = float("nan")
    run(ctx, y, rng.integers(0, classes, (6, 2)), n, None, 10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [33, 900, 4100, 40000])
def test_rows_without_a_distribution_and_extreme_values(ctx, dtype, classes):
    rng = np.random.default_rng(classes + 3)
    x = logits(rng, 12, classes, dtype)
    x[0, classes // 2] = float("nan")
    x[1, classes - 1] = float("inf")
    x[2] = -float("inf")
    x[3] = LOWEST[dtype]                        # the type's lowest value: allowed, and uniform
    x[4] = LOWEST[dtype]
    x[4, 7] = 0.0
    x[5, 3] = -LOWEST[dtype]                    # differences beyond the type's range
    x[5, 4] = LOWEST[dtype]
    x[6] = 0.0                                  # zeros of both signs are equal
    x[6, 1::2] = -0.0
    x[7] = 3.5
    x[8] = -float("inf")
    x[8, classes - 1] = -2.0
    x[9, :] = float("nan")
    x[10, 0], x[10, 1] = float("inf"), -float("inf")
    given = np.stack([np.array([classes // 2, classes - 1, 7, 3, 4, 0, 1]) for _ in range(12)])
    run(ctx, x, given, top=32)
    run(ctx, x, given, top=1, temperature=0.01)
    run(ctx, x, given, top=6, temperature=100.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [64, 1500, 9000, 131072])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "two values", "steps"])
def test_orders_that_meet_the_selection_worst(ctx, dtype, classes, order):
    c = torch.arange(classes, dtype=torch.float64)
    v = {"rising": c / classes * 8, "falling": -c / classes * 8, "equal": 0 * c, "two values": (c % 7 == 3).double(), "steps": torch.floor(c / 97) % 50}[order]
    x = v.to(DT[dtype]).cuda().repeat(3, 1).contiguous()
    given = np.array([[0, classes - 1, classes // 2]] * 3)
    for top in (1, 7, 32):
        run(ctx, x, given, top=top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,classes", [(3, 8192), (3, 9000), (500, 20000), (1, 1 << 20)])
@pytest.mark.parametrize("few", [512, 1024, 2048, 3000])
def test_equal_classes_where_few_come_first(ctx, dtype, rows, classes, few):
    """The first classes hold a few better ones and no equals; all the others are equal, so the lowest numbers among them are the answer."""
    x = torch.full((rows, classes), 5.0, dtype=DT[dtype], device="cuda")
    x[:, :few] = 4.0
    for top in (2, 10, 32):
        x[:, : 16 * ((top + 3) // 4) : 16] = 6.0
        run(ctx, x, np.array([[0, few - 1, few, classes - 1]] * rows), top=top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,classes", [(1, 16384), (1, 16385), (128, 16385), (147, 20481), (147, 61441), (341, 61441), (342, 61441), (341, 8193), (341, 28673), (2047, 2049), (2048, 2049), (204, 2049), (205, 2049),
                                          (2048, 2700)])
def test_sizes_where_the_work_is_dealt_out_differently(ctx, dtype, rows, classes):
    rng = np.random.default_rng(rows + classes)
    for given, top in ((2, 6), (5, 12)):
        run(ctx, logits(rng, rows, classes, dtype, scale=1.0), rng.integers(0, classes, (rows, given)), n=rng.integers(0, classes + 1, rows), top=top)


@pytest.mark.parametrize("rows", [1, 2, 7, 40, 300, 1500])
def test_numbers_of_rows(ctx, rows):
    """From rows that many workgroups share to rows by the thousand; outputs and scratch used again by other calls."""
    rng = np.random.default_rng(rows)
    out = mt.alloc_scores(rows, 2, 8)
    for classes in (3000, 50, 20000 if rows < 100 else 700, 3000):
        x = logits(rng, rows, classes, "f32")
        run(ctx, x, rng.integers(0, classes, (rows, 2)), top=8, out=out)
    small = mt.alloc_scores(max(1, rows // 2), 2, 8)
    small.scratch = out.scratch
    x = logits(rng, small.entropy.shape[0], 9000 if rows < 100 else 900, "bf16")
    run(ctx, x, rng.integers(0, 900, (x.shape[0], 2)), top=8, out=small)


def test_outputs_alone(ctx):
    """Each output without the others, through the argument block."""
    rng = np.random.default_rng(1)
    from paper_1901_06887_amd import binding as B
    x = logits(rng, 4, 5000, "f32")
    given = torch.from_numpy(rng.integers(0, 5000, (4, 2)).astype(np.int32)).cuda()
    full = mt.alloc_scores(4, 2, 5)
    mt.score(ctx, x, full, given=given)
    for name in ("given_logprobs", "given_ranks", "entropy", "top_ids", "top_logprobs"):
        want = getattr(full, name)
        got = torch.full_like(want, 77)
        a = B.mt_score_args()
        a.logits, a.rows, a.classes, a.row_stride, a.temperature = x.data_ptr(), 4, 5000, 5000, 1.0
        a.scratch, a.scratch_bytes = full.scratch.data_ptr(), full.scratch.numel()
        if name.startswith("given"):
            a.given, a.n_given = given.data_ptr(), 2
        if name.startswith("top"):
            a.top = 5
        setattr(a, name, got.data_ptr())
        ctx.score(torch.cuda.current_stream().cuda_stream, a)
        assert torch.equal(got, want), name


def test_outputs_of_a_run(ctx):
    """The logits and class counts of mt_run, as they come."""
    rng = np.random.default_rng(12)
    worker = mt.Context(3, 64, 64, 300, 4 << 20, mt.MT_F32, 0)
    for t, n in enumerate((10, 300, 77)):
        worker.register_model(t, [mt.layer_spec(mt.MT_FC, mt.MT_ACT_NONE, 64, n)], [rng.standard_normal((n, 64)).astype(np.float32)], [None])
    ids = torch.from_numpy(np.array([0, 1, 2, 1, 5, 0], dtype=np.int32)).cuda()         # 5: no such tenant
    served = mt.serve(worker, ids, torch.from_numpy(rng.standard_normal((6, 64)).astype(np.float32)).cuda())
    o = mt.alloc_scores(6, 0, 3)
    mt.score(worker, served.logits, o, n_classes=served.n_classes)
    ref = lm.scored(served.logits.double().cpu().numpy(), served.n_classes.cpu().numpy(), top=3)
    agree(o, ref, 0, 3)
    assert torch.equal(o.top_ids[:, 0], served.labels)
    worker.close()


def test_offsets_past_32_bits(ctx):
    stride = (1 << 31) + 12
    buf = torch.empty(2 * stride + 5000, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 5000), (stride, 1))
    x.copy_(torch.randn(3, 5000))
    run(ctx, x, np.array([[1], [2], [4999]]), top=4)


def test_more_rows_than_a_grid_of_threads(ctx):
    rows, classes = (2 << 21) + 3, 40
    x = torch.randn(rows, classes, device="cuda").to(torch.bfloat16)
    given = torch.randint(0, classes, (rows, 2), dtype=torch.int32, device="cuda")
    n = torch.randint(0, classes + 1, (rows,), dtype=torch.int32, device="cuda")
    allowed = torch.randint(-(1 << 31), 1 << 31, (rows, 2), dtype=torch.int64, device="cuda").to(torch.int32)
    o = mt.alloc_scores(rows, 2, 3)
    mt.score(ctx, x, o, given=given, n_classes=n, allowed=allowed)
    torch.cuda.synchronize()
    for first in (0, (1 << 21) - 5, (2 << 21) - 5, rows - 8):
        few = slice(first, first + 8)
        ref = lm.scored(x[few].double().cpu().numpy(), n[few].cpu().numpy(), allowed[few].cpu().numpy().view(np.uint32), given[few].cpu().numpy(), 3)
        agree(mt.Scores(o.given_logprobs[few], o.given_ranks[few], o.entropy[few], o.top_ids[few], o.top_logprobs[few], o.scratch), ref, 2, 3)
    c = torch.arange(classes, device="cuda")
    ok = (c < n[:, None]) & ((allowed[:, c // 32] >> (c % 32)) & 1).bool()
    assert bool(((o.top_ids >= 0).sum(1) == ok.sum(1).clamp(max=3)).all())
    assert torch.equal(o.top_ids[:, 0].long(), torch.where(ok.any(1), torch.where(ok, x.double(), -1e300).argmax(1), -1))


def test_streams_and_graphs(ctx):
    rng = np.random.default_rng(3)
    xs = [logits(rng, 2, 60000, "bf16") for _ in range(4)]
    given = torch.from_numpy(rng.integers(0, 60000, (2, 1)).astype(np.int32)).cuda()
    outs, streams = [mt.alloc_scores(2, 1, 20) for _ in xs], [torch.cuda.Stream() for _ in xs]
    wants = []
    for x in xs:
        o = mt.alloc_scores(2, 1, 20)
        wants.append(mt.score(ctx, x, o, given=given))
    torch.cuda.synchronize()
    for _ in range(5):
        for x, o, s in zip(xs, outs, streams):
            mt.score(ctx, x, o, given=given, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, wants):
        assert all(torch.equal(getattr(o, k), getattr(w, k)) for k in ("given_logprobs", "given_ranks", "entropy", "top_ids", "top_logprobs"))
    o, x = outs[0], xs[0].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mt.score(ctx, x, o, given=given)
    for i in range(4):
        x.copy_(xs[i])
        o.entropy.zero_(), o.top_ids.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(o, k), getattr(wants[i], k)) for k in ("given_logprobs", "given_ranks", "entropy", "top_ids", "top_logprobs")), i


def test_no_rows(ctx):
    mt.score(ctx, torch.empty(0, 10, device="cuda"), mt.alloc_scores(0, 0, 3))


def test_refusals_of_tensors(ctx):
    x = torch.zeros(4, 50, device="cuda")
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    o = mt.alloc_scores(4, 2, 3)
    for args, kw in (((x.half(), o), dict(given=ids)), ((x[:3], o), dict(given=ids)), ((x, o), {}), ((x, o), dict(given=ids.long())), ((x, o), dict(given=ids[:, :1])),
                     ((x, o), dict(given=ids, n_classes=torch.zeros(4, dtype=torch.int64, device="cuda"))), ((x, o), dict(given=ids, allowed=ids[:, :1])),
                     ((x, mt.alloc_scores(4, 0, 3)), dict(given=ids)), ((x.cpu(), o), dict(given=ids)), ((x.t().contiguous().t(), o), dict(given=ids))):
        with pytest.raises(ValueError):
            mt.score(ctx, *args, **kw)
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        with pytest.raises(mt.MtError) as e:
            mt.score(ctx, x, o, given=ids, temperature=t)
        assert e.value.status == 1
    for kw in (dict(n_given=17), dict(top=33)):
        with pytest.raises(mt.MtError):
            mt.alloc_scores(4, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_temperatures_whose_multiples_leave_the_range_are_refused(ctx, dtype):
    """Below 2^-126 a temperature's reciprocal, or twice of it, is beyond fp32's range or near it: refused, and 2^-126 itself is not."""
    x = logits(np.random.default_rng(0), 3, 100, dtype)
    o = mt.alloc_scores(3, 0, 2)
    for t in (2.0 ** -126 * (1 - 2.0 ** -23), 6e-39, 4e-39, 3e-39, 1e-39):
        with pytest.raises(mt.MtError) as e:
            mt.score(ctx, x, o, temperature=t)
        assert e.value.status == 1, t
    run(ctx, x, np.array([[0, 99]] * 3), top=5, temperature=2.0 ** -126)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("classes", [33, 900, 4100, 40000])
def test_temperatures_of_the_whole_range(ctx, dtype, classes):
    """At temperatures of the size of the largest differences these count, however large; at the smallest temperatures the smallest differences do."""
    rng = np.random.default_rng(classes + 4)
    x = logits(rng, 8, classes, dtype)
    x[0, ::2], x[0, 1::2] = LOWEST[dtype], -LOWEST[dtype]          # as far apart as there is
    x[1] = LOWEST[dtype]
    x[1, 5] = -LOWEST[dtype]
    x[2] = -LOWEST[dtype]
    x[2, 7] = LOWEST[dtype]
    x[3] = torch.from_numpy(rng.uniform(-3e38, 3e38, classes)).to(DT[dtype])
    x[4, ::3] = -float("inf")
    x[5] = torch.from_numpy(rng.integers(-64, 64, classes) * 2.0 ** -130).to(DT[dtype])
    x[6] = torch.from_numpy(rng.integers(-64, 64, classes) * 2.0 ** -128).to(DT[dtype])
    given = np.array([[0, 1, 5, 7, classes - 1]] * 8)
    for temperature in (1e38, 3.4e38, 1e36, 1e30, 1e20, 1e-20, 2e-38, 2.0 ** -126):
        run(ctx, x, given, top=9, temperature=temperature)


def test_outputs_on_tensors_alone(ctx):
    """An output that is None is left out; the others are as they were."""
    rng = np.random.default_rng(2)
    x = logits(rng, 4, 5000, "f32")
    given = torch.from_numpy(rng.integers(0, 5000, (4, 2)).astype(np.int32)).cuda()
    names = ("given_logprobs", "given_ranks", "entropy", "top_ids", "top_logprobs")
    full = mt.score(ctx, x, mt.alloc_scores(4, 2, 5), given=given)
    for kept in [(n,) for n in names] + [("given_logprobs", "top_logprobs"), ("given_ranks", "top_ids"), ("entropy", "top_logprobs")]:
        o = mt.alloc_scores(4, 2, 5)
        for n in names:
            getattr(o, n).fill_(77) if n in kept else setattr(o, n, None)
        mt.score(ctx, x, o, given=given if any(n.startswith("given") for n in kept) else None)
        for n in kept:
            assert torch.equal(getattr(o, n), getattr(full, n)), (kept, n)
    # outputs without what they are for, or of other sizes than each other
    for change in (dict(given_logprobs=torch.empty(4, 3, device="cuda")), dict(top_logprobs=torch.empty(4, 6, device="cuda")), dict(given_ranks=None, given_logprobs=None)):
        o = mt.alloc_scores(4, 2, 5)
        for n, v in change.items():
            setattr(o, n, v)
        with pytest.raises(ValueError):
            mt.score(ctx, x, o, given=given)
    o = mt.alloc_scores(4, 2, 5)
    o.given_ranks = None
    with pytest.raises(ValueError):
        mt.score(ctx, x, o)
