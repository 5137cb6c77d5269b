"""mt_sample against whole-number weights from 64-bit exponentials."""
import numpy as np
import pytest
import torch

import lm_cache_common as lc
import paper_1901_06887_amd as mt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = mt.Context(1, 1, 64, 1, 1 << 16, mt.MT_BF16, 0)
    yield c
    c.close()


def floats(v):
    return torch.tensor(np.asarray(v, dtype=np.float32), device="cuda")


def whole(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda")


def check(ctx, x, u, n=None, allowed=None, out=None, **kw):
    """x: logits on the device; settings: lists of a value a row."""
    R, C = x.shape
    o = mt.alloc_samples(R, C) if out is None else out
    mt.sample(ctx, x, floats(u), o, n_classes=None if n is None else whole(n), allowed=None if allowed is None else torch.from_numpy(allowed.view(np.int32)).cuda(),
              **{k: whole(v) if k == "top_k" else floats(v) for k, v in kw.items()})
    v = lc.in_64(x)
    for r in range(R):
        one = {k: w[r] if k == "top_k" else np.float32(w[r]) for k, w in kw.items()}
        want = lc.sampled(v[r], np.float32(u[r]), n=None if n is None else n[r], allowed=None if allowed is None else allowed[r], **one)
        got = (int(o.ids[r]), float(o.logprobs[r]), int(o.kept[r]))
        assert got[0] == want[0] and got[2] == want[2], (r, got, want, one)
        if np.isfinite(want[1]):
            assert abs(got[1] - want[1]) <= 2.0 ** -23 * abs(want[1]) + 2.0 ** -30, (r, got, want)         # (rounded once)
        else:
            assert np.isnan(got[1]) == np.isnan(want[1]) and (np.isnan(got[1]) or got[1] == want[1]), (r, got, want)
    return o


def logits(rng, R, C, dtype, peak=9.0):
    x = 2.5 * rng.standard_normal((R, C), dtype=np.float32) + peak * (rng.random((R, C)) < 4.0 / C).astype(np.float32)
    return torch.from_numpy(x).to(lc.DTYPES[dtype]).cuda()


SIZES = [1, 2, 7, 64, 257, 1000, 4095, 4097, 10000, 32768, 65001, 131072]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", SIZES)
def test_settings_of_every_row(ctx, dtype, C):
    rng = np.random.default_rng(C)
    settings = [dict(), dict(top_k=1), dict(top_k=50), dict(top_k=3000), dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.05), dict(min_p=1.0), dict(top_k=40, top_p=0.8), dict(top_k=200, min_p=0.01, top_p=0.95),
                dict(min_p=0.001, top_p=0.5), dict(temperature=0.0), dict(temperature=0.1, top_p=0.99), dict(temperature=5.0), dict(temperature=3.0, top_p=0.9999), dict(top_p=0.0), dict(top_p=1.0, top_k=C),
                dict(top_k=-5, min_p=-1.0, top_p=7.0), dict(top_k=C - 1), dict(min_p=3.0)]
    R = len(settings)
    column = lambda key, default: [s.get(key, default) for s in settings]  # noqa: E731
    x = logits(rng, R, C, dtype)
    for u in (rng.random(R), np.zeros(R), np.full(R, 1 - 2.0 ** -24)):
        check(ctx, x, u, temperature=column("temperature", 1.0), top_k=column("top_k", 0), top_p=column("top_p", 1.0), min_p=column("min_p", 0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [31, 1000, 33000])
@pytest.mark.parametrize("key,value", [("top_k", 20), ("top_p", 0.7), ("min_p", 0.02), ("temperature", 0.8)])
def test_one_setting_alone(ctx, dtype, C, key, value):
    rng = np.random.default_rng(C)
    check(ctx, logits(rng, 9, C, dtype), rng.random(9), **{key: [value] * 9})
    check(ctx, logits(rng, 9, C, dtype), rng.random(9))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [40, 3001, 65001])
def test_masks_and_class_counts(ctx, dtype, C):
    rng = np.random.default_rng(C)
    R = 10
    allowed = rng.integers(0, 1 << 32, (R, -(-C // 32) + 1), dtype=np.uint32)
    allowed[1] = 0
    allowed[2] = 0
    allowed[2, (C - 1) // 32] = 1 << ((C - 1) % 32)
    n = [C, C, C, 0, -3, C + 9, 1, C // 2, C - 1, C]
    x = logits(rng, R, C, dtype)
    x[7, C // 2:] = float("nan")                     # (behind the classes that there are)
    x[8, :C // 3] = -float("inf")
    x[9] = -float("inf")
    for kw in (dict(), dict(top_k=[5] * R), dict(top_p=[0.8] * R), dict(top_k=[100] * R, top_p=[0.9] * R, min_p=[0.01] * R)):
        check(ctx, x, rng.random(R), n=n, allowed=allowed, **kw)
        check(ctx, x, rng.random(R), n=n, **kw)
        check(ctx, x, rng.random(R), allowed=np.where(np.arange(R)[:, None] == 7, 0, allowed).astype(np.uint32), **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [50, 5000, 40001])
def test_ties(ctx, dtype, C):
    """Equal logits: lower numbers first, whole rows of them, and both zeros."""
    rng = np.random.default_rng(C)
    x = torch.zeros(8, C)
    x[0, ::2] = -0.0
    x[1] = torch.from_numpy(rng.integers(0, 3, C).astype(np.float32))
    x[2] = torch.from_numpy(rng.integers(0, 40, C).astype(np.float32) / 4)
    x[3, C - 1] = 1
    x[4] = -1e30
    x[5] = torch.from_numpy(np.where(rng.random(C) < 0.5, 2.0, -2.0).astype(np.float32))
    x[6, C // 2:] = 1e-3
    x[7] = 88.0
    x = x.to(lc.DTYPES[dtype]).cuda()
    for kw in (dict(), dict(top_k=[7] * 8), dict(top_k=[C // 2 + 1] * 8), dict(top_p=[0.25] * 8), dict(top_k=[C - 3] * 8, top_p=[0.5] * 8), dict(min_p=[0.5] * 8), dict(temperature=[0.0] * 8), dict(temperature=[1e-3] * 8, top_p=[0.4] * 8)):
        check(ctx, x, rng.random(8), **kw)


@pytest.mark.parametrize("C", [100, 70000])
def test_odd_rows_and_settings(ctx, C):
    rng = np.random.default_rng(C)
    x = logits(rng, 12, C, "f32")
    x[0, C - 1], x[1, 3], x[2, 5] = float("nan"), float("inf"), -float("nan")
    x[3, 7] = 3e38
    x[4] = -3e38
    x[4, C // 2] = 3e38
    nan, inf = float("nan"), float("inf")
    u = [0.5, 0.5, 0.5, 0.5, 0.5, nan, 1.0, 2.5, -1.0, 0.3, 0.3, 0.3]
    check(ctx, x, u)
    check(ctx, x, [0.4] * 12, temperature=[1, 1, 1, 1, 1, nan, -1.0, inf, 2.0 ** -126, 1e-40, 3e38, 0.0])
    check(ctx, x, [0.4] * 12, top_p=[0.9] * 5 + [nan, -1.0, 1e-30, inf, -inf, 1 - 2.0 ** -24, 0.5], top_k=[3] * 6 + [0] * 6)
    check(ctx, x, [0.4] * 12, min_p=[0.1] * 5 + [nan, -1.0, 1e-30, inf, -inf, 1 - 2.0 ** -24, 0.5])
    check(ctx, x, [0.7] * 12, temperature=[1e30] * 12, top_p=[0.5] * 12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_left_out_outputs(ctx, dtype):
    rng = np.random.default_rng(7)
    wide = logits(rng, 5, 3010, dtype)
    x = wide[:, 3:3004]
    u = rng.random(5)
    whole_out = check(ctx, x, u, top_p=[0.9] * 5)
    for left in ("ids", "logprobs", "kept"):
        o = mt.alloc_samples(5, 3001)
        setattr(o, left, None)
        mt.sample(ctx, x, floats(u), o, top_p=floats([0.9] * 5))
        for name in ("ids", "logprobs", "kept"):
            if name != left:
                assert torch.equal(getattr(o, name), getattr(whole_out, name))


def test_shares_of_many_draws(ctx):
    """Over a fine grid of random numbers every class comes as often as its weight says, to one draw."""
    rng = np.random.default_rng(11)
    R, C = 2000, 300
    x = logits(rng, 1, C, "f32").expand(R, C).contiguous()
    o = mt.alloc_samples(R, C)
    mt.sample(ctx, x, floats((np.arange(R) + 0.5) / R), o, top_p=floats([0.95] * R))
    counts = np.bincount(o.ids.cpu().numpy(), minlength=C)
    lp = {int(i): float(v) for i, v in zip(o.ids, o.logprobs)}
    assert all(abs(counts[c] - R * np.exp(v)) <= 1.01 for c, v in lp.items()) and abs(sum(np.exp(v) for v in lp.values()) - 1) < (int(o.kept[0]) + 1) / R


def test_captured_replayed_and_on_two_streams(ctx):
    rng = np.random.default_rng(12)
    R, C = 3, 131072
    x, u, p, k = logits(rng, R, C, "bf16"), floats(rng.random(R)), floats([0.9, 1.0, 0.5]), whole([0, 50, 0])
    outs = [mt.alloc_samples(R, C) for _ in range(3)]
    outs[1].scratch = outs[0].scratch
    run = lambda o, **kw: mt.sample(ctx, x, u, o, top_p=p, top_k=k, **kw)  # noqa: E731
    run(outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(outs[0])
    side = torch.cuda.Stream()
    for again in range(4):
        x.copy_(logits(rng, R, C, "bf16")), u.copy_(floats(rng.random(R)))
        torch.cuda.synchronize()
        graph.replay()
        run(outs[2], stream=side)
        run(outs[1])
        torch.cuda.synchronize()
        v = lc.in_64(x)
        for r in range(R):
            want = lc.sampled(v[r], np.float32(u[r].item()), top_p=np.float32(p[r].item()), top_k=int(k[r]))
            for o in outs:
                assert int(o.ids[r]) == want[0] and int(o.kept[r]) == want[2]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", [(3, 131072), (300, 20000), (40, 3000)])
def test_results_do_not_depend_on_timing(ctx, dtype, R, C):
    rng = np.random.default_rng(R)
    x, u = logits(rng, R, C, dtype), floats(rng.random(R))
    p, k, m = floats(rng.choice([1.0, 0.95, 0.5], R)), whole(rng.choice([0, 0, 40, 700], R)), floats(rng.choice([0.0, 0.0, 0.01], R))
    outs = [mt.alloc_samples(R, C) for _ in range(6)]
    for o in outs:
        mt.sample(ctx, x, u, o, top_p=p, top_k=k, min_p=m)
    for o in outs[1:]:
        assert torch.equal(o.ids, outs[0].ids) and torch.equal(o.kept, outs[0].kept) and torch.equal(o.logprobs, outs[0].logprobs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_that_no_bin_suits(ctx, dtype):
    """Masks of the type's lowest value, a few logits far in front, many equal ones in a narrow band, all settings."""
    rng = np.random.default_rng(21)
    C = 20000
    x = 2.5 * rng.standard_normal((6, C), dtype=np.float32)
    x[0, rng.random(C) < 0.95] = np.finfo(np.float32).min if dtype == "f32" else -3.38e38
    x[1, :3] = 1e4
    x[2] = 5.0 + 1e-4 * x[2]
    x[3, rng.random(C) < 0.5] = 7.0
    x[4] *= 1e-30
    x[5] *= 1e6
    t = torch.from_numpy(x).to(lc.DTYPES[dtype]).cuda()
    for kw in (dict(), dict(top_p=[0.9] * 6), dict(top_k=[100] * 6), dict(top_k=[5000] * 6, top_p=[0.7] * 6), dict(min_p=[0.5] * 6, top_p=[0.6] * 6)):
        check(ctx, t, rng.random(6), **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [700, 33000])
def test_nearly_all_of_the_weight(ctx, dtype, C):
    """Bars far below the middle of a row, at temperatures that make it flat or steep."""
    rng = np.random.default_rng(C + 1)
    top_p = [0.99, 0.9901, 0.999, 1 - 2.0 ** -14, 1 - 2.0 ** -19, 1 - 2.0 ** -24] * 3
    x = logits(rng, 18, C, dtype)
    check(ctx, x, rng.random(18), top_p=top_p, temperature=[0.6] * 6 + [1.0] * 6 + [6.0] * 6)
    check(ctx, x, rng.random(18), top_p=top_p, min_p=[1e-6] * 18)


def test_many_rows(ctx):
    """The rows of a large batch, few of them looked at one by one."""
    rng = np.random.default_rng(13)
    R, C = 5000, 500
    x, u = logits(rng, R, C, "bf16"), rng.random(R)
    o = mt.alloc_samples(R, C)
    mt.sample(ctx, x, floats(u), o, top_k=whole([30] * R), top_p=floats([0.9] * R))
    v = lc.in_64(x)
    for r in (*range(0, R, 37), R - 1):
        want = lc.sampled(v[r], np.float32(u[r]), top_k=30, top_p=np.float32(0.9))
        assert int(o.ids[r]) == want[0] and int(o.kept[r]) == want[2]
    assert mt.sample(ctx, x[:0], floats([]), mt.alloc_samples(0, C)).ids.numel() == 0


def test_calls_on_tensors_refuse(ctx):
    x, o = torch.zeros(4, 10, device="cuda"), mt.alloc_samples(4, 10)
    f = floats([0.5] * 4)
    for args, kw in (((x.half(), f), {}), ((x, f[:3]), {}), ((x, None), {}), ((x, f.double()), {}), ((x[0], f), {}), ((x.t(), floats([0.5] * 10)), {}), ((x, f), dict(temperature=f[:2])), ((x, f), dict(top_k=f)),
                     ((x, f), dict(top_p=whole([1] * 4))), ((x, f), dict(min_p=f.cpu())), ((x, f), dict(n_classes=f)), ((x, f), dict(allowed=whole([1] * 4).view(4, 1)[:, :0]))):
        with pytest.raises(ValueError):
            mt.sample(ctx, *args, o, **kw)
    o.ids = o.logprobs = o.kept = None
    with pytest.raises(mt.MtError):
        mt.sample(ctx, x, f, o)
