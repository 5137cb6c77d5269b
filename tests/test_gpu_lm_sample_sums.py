"""mt_sample where a row's small weights, each next to nothing of the largest, decide."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_1901_06887_amd as mt
from test_gpu_lm_sample import ctx, floats, whole  # noqa: F401

pytestmark = pytest.mark.gpu

OFF = 2.0 ** -39             # of a weight, of a sum


def settle(few, far, many, top_p, u):
    """(kept, weight in front of the draw, all) of `few` classes of weight 1 and `many` of weight e^far, exactly but for that weight's double."""
    w = Fraction(float(np.exp(np.float64(far))))
    target, total = Fraction(float(np.float32(top_p))) * (few + many * w), few + many * w
    kept = max(-(-target // 1), 1) if target <= few else min(few + -(-(target - few) // w), few + many)
    return int(kept), Fraction(float(np.float32(u))) * (min(kept, few) + max(kept - few, 0) * w), w, total


@pytest.mark.parametrize("C", [1 << 20, 131072, 33000, 8192, 5000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_small_weights_of_one_size(ctx, dtype, C):
    """One class of weight 1, or three, in front of thousands of equal ones that no list holds: how many are kept goes by their sum, however little each weighs."""
    rng = np.random.default_rng(C)
    rows = []
    for few, far in ((1, -29.875), (1, -26.0), (3, -20.0), (1, -35.0), (2, -8.0), (1, -40.0)):
        tail = (C - few) * np.exp(far) / few
        for part in (0.5, 0.25, 0.9):
            rows.append((few, far, 1 - tail / (1 + tail) * part))
    # (top_p has 24 bits: rows where that leaves nothing but all or the first are left out)
    rows = [(few, far, np.float32(p)) for few, far, p in rows if p < 1 - 2.0 ** -25]
    assert len(rows) >= (9 if C > 10000 else 6)
    x = np.empty((len(rows), C), np.float32)
    places = []
    for i, (few, far, _) in enumerate(rows):
        x[i] = far
        places.append(np.sort(rng.choice(C, few, replace=False)))
        x[i, places[-1]] = 0
    t = torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    assert np.array_equal(t.float().cpu().numpy(), x)
    for u in (0.3, 1 - 2.0 ** -24, 0.9999):
        o = mt.alloc_samples(len(rows), C)
        mt.sample(ctx, t, floats([u] * len(rows)), o, top_p=floats([p for _, _, p in rows]))
        for i, (few, far, p) in enumerate(rows):
            kept, front, w, total = settle(few, far, C - few, p, u)
            # a class counts w: so many of them lie in what sums are off (target and prefix: twice)
            near = 2 * OFF * float(total / w) + 1
            assert abs(int(o.kept[i]) - kept) <= near, (rows[i], int(o.kept[i]), kept, near)
            # the draw: classes in their order, few of weight 1 among those of weight w (kept ones are the first of either)
            c, heavy = int(o.ids[i]), places[i][:min(kept, few)]
            before = int(np.searchsorted(places[i], c))
            low = min(before, len(heavy)) + min(c - before, max(kept - few, 0)) * w
            assert c not in places[i] or c in heavy
            high = low + (1 if c in places[i] else w)
            slack = Fraction(2 * OFF + 2.0 ** -45) * total + w
            assert low - slack <= front < high + slack, (rows[i], u, c, float(low), float(front), float(high))
            assert abs(float(o.logprobs[i]) - float(np.log(float((1 if c in places[i] else w) / (min(int(o.kept[i]), few) + max(int(o.kept[i]) - few, 0) * w))))) <= 2.0 ** -22 * 45


def test_the_row_whose_weights_vanished(ctx):
    """2^20 classes, one of weight 1, the others 2^-43.1 each: all but 2^-24 of the weight are half of these, not the first class alone."""
    C = 1 << 20
    x = torch.full((1, C), -29.875, device="cuda")
    x[0, 77] = 0
    o = mt.alloc_samples(1, C)
    mt.sample(ctx, x, floats([0.5]), o, top_p=floats([1 - 2.0 ** -24]))
    kept, _, w, total = settle(1, -29.875, C - 1, 1 - 2.0 ** -24, 0.5)
    assert kept > 400000 and abs(int(o.kept[0]) - kept) <= 2 * OFF * float(total / w) + 1 and int(o.ids[0]) == 77


@pytest.mark.parametrize("C", [20000, 65001])
def test_settings_together_settled_digit_by_digit(ctx, C):
    """top_k of thousands, min_p and top_p over small weights of many sizes."""
    rng = np.random.default_rng(C)
    R = 8
    x = (-22.0 - 3.0 * rng.random((R, C))).astype(np.float32)
    x[:, 5] = 0
    order = np.argsort(-x.astype(np.float64), axis=1, kind="stable")
    z = np.take_along_axis(x.astype(np.float64), order, 1)
    w = np.exp(z)
    top_k, min_p = C - 3000, np.float32(np.exp(-24.5))
    keep = np.minimum(top_k, (w >= float(min_p)).sum(1))
    top_p = np.float32(1 - 2.0 ** -24 * np.array([64, 128, 3, 5, 17, 100, 7, 30.0]))
    o = mt.alloc_samples(R, C)
    mt.sample(ctx, torch.from_numpy(x).cuda(), floats([0.1] * R), o, top_p=floats(top_p), top_k=whole([top_k] * R), min_p=floats([min_p] * R))
    for r in range(R):
        sums = np.cumsum(w[r, :keep[r]].astype(np.longdouble))
        kept = int(np.searchsorted(sums, np.longdouble(top_p[r]) * sums[-1])) + 1
        near = 2 * OFF * float(sums[-1] / w[r, kept - 1]) + 1
        assert abs(int(o.kept[r]) - kept) <= near and near < 20, (r, int(o.kept[r]), kept, near)
        assert int(o.ids[r]) == 5


def test_calls_without_a_scratch(ctx):
    x = torch.randn(3, 70000, device="cuda")
    outs = [mt.alloc_samples(3, 70000) for _ in range(3)]
    outs[1].scratch, outs[2].scratch = None, torch.full((5,), 7, dtype=torch.uint8, device="cuda")
    for o in outs:
        mt.sample(ctx, x, floats([0.3, 0.6, 0.9]), o, top_p=floats([0.9] * 3))
    assert all(torch.equal(o.ids, outs[0].ids) and torch.equal(o.kept, outs[0].kept) for o in outs) and torch.all(outs[2].scratch == 7)
    for bad in (torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.uint8), "x"):
        outs[1].scratch = bad
        with pytest.raises(ValueError):
            mt.sample(ctx, x, floats([0.3] * 3), outs[1])
