"""mt_kv_copy: long lists, and pages that stand in both lists."""
import numpy as np
import pytest
import torch

import lm_cache_common as lc
import paper_1901_06887_amd as mt
from test_gpu_lm_pages import Pair, ctx, ints  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("n", [4095, 4096, 4097, 20000, 300000])
def test_long_lists(ctx, kv8, n):
    """Of the pairs with one target the last counts, and counts for nothing where it is out of range or names its own page; on either side of the length from which pairs are looked up."""
    rng = np.random.default_rng(n)
    p = Pair(ctx, 3000, 16, 2, 4, kv8, heads=2, dim=16, layers=2)
    src, dst = rng.integers(-3, 1500, n), rng.integers(1500, 3010, n)
    src[rng.random(n) < 0.01], dst[rng.random(n) < 0.01] = 3000, -1
    own = np.nonzero(rng.random(n) < 0.01)[0]
    src[own] = dst[own]
    if n == 20000:
        src[-1], dst[-1], src[0], dst[0] = 7, 2999, 5, 1500
    last = {int(d): int(s) for s, d in zip(src, dst) if 0 <= d < 3000}
    assert len(last) > 1000
    before = [x.clone() for x in p.original]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = ints(src), ints(dst)
    torch.cuda.synchronize()
    for again in range(2):
        mt.kv_copy(ctx, p.c, a, b, stream=side if again else None)
        torch.cuda.synchronize()
    moves = [(s, d) for d, s in last.items() if 0 <= s < 3000 and s != d]
    at, of = (torch.tensor(m).cuda() for m in zip(*((d, s) for s, d in moves)))
    for x, was in zip(p.parts, before):
        was[:, at] = was[:, of]
        assert torch.equal(x.view(torch.uint8), was)
    assert int(p.c.refs.sum()) == 0


def test_long_lists_captured(ctx):
    p = Pair(ctx, 200, 16, 2, 4)
    a, b = ints([0] * 6000), ints([199] * 6000)
    mt.kv_copy(ctx, p.c, a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.kv_copy(ctx, p.c, a, b)
    for again in range(4):
        src, dst = np.arange(6000) * (again + 3) % 100, 100 + np.arange(6000) * 7 % 100
        a.copy_(ints(src)), b.copy_(ints(dst))
        was = [x.view(torch.uint8).clone() for x in p.parts]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        last = dict(zip(dst.tolist(), src.tolist()))
        for x, w in zip(p.parts, was):
            w[:, list(last)] = w[:, list(last.values())]
            assert torch.equal(x.view(torch.uint8), w)
        mt.kv_free(ctx, p.c, ints([0]))
        mt.kv_compact(ctx, p.c)                     # (the same work memory)


@pytest.mark.parametrize("n", [2, 5000])
def test_pages_in_both_lists(ctx, n):
    """a over b and b over c: b is a; c is bit for bit of what b was before or behind; nothing else changes."""
    p = Pair(ctx, 12, 256, 2, 4, True, heads=4, dim=128, layers=2)
    src, dst = [1] * (n - 1) + [2], [2] * (n - 1) + [3]
    mt.kv_copy(ctx, p.c, ints(src), ints(dst))
    for x, was in zip(p.parts, p.original):
        x = x.view(torch.uint8)
        assert torch.equal(x[:, 2], was[:, 1]) and torch.all((x[:, 3] == was[:, 1]) | (x[:, 3] == was[:, 2]))
        rest = [i for i in range(12) if i not in (2, 3)]
        assert torch.equal(x[:, rest], was[:, rest])
