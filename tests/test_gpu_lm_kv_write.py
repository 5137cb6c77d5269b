"""mt_kv_write against whole numbers and 64-bit rounding."""
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


def ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda")


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def written(before, c, table, dtype, kv8, rows, layer):
    """What the cache holds behind a call: before (k, v, k_scales, v_scales as bytes), with rows (sequence, token, k, v) in their places."""
    k, v, ks, vs = (None if b is None else b.copy() for b in before)
    page = c.k.shape[3]
    es = c.k.element_size()
    for s, t, kr, vr in rows:
        p, slot = table[s, t // page], t % page
        for row, to, scales, turned in ((kr, k, ks, False), (vr, v, vs, True)):
            if kv8:
                q, e = lc.in_8_bits(lc.in_64(row))
                scales[layer, p, :, slot] = e
                q = q[..., None]
            else:
                q = bits(row).reshape(row.shape[0], row.shape[1], es)
            if turned:
                to.reshape(*c.v.shape, es)[layer, p, :, :, slot] = q
            else:
                to.reshape(*c.k.shape, es)[layer, p, :, slot] = q
    return k, v, ks, vs


def held(c):
    return [None if x is None else bits(x) for x in (c.k, c.v, c.k_scales, c.v_scales)]


def same(a, b):
    for x, y in zip(a, b):
        assert (x is None) == (y is None)
        if x is not None:
            assert np.array_equal(x, y)


KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("heads,dim,page,layers", [(1, 16, 16, 1), (3, 80, 32, 2), (8, 128, 64, 1), (2, 256, 128, 3), (5, 144, 256, 1)])
@pytest.mark.parametrize("what", ["step", "ragged"])
def test_rows_and_nothing_else(ctx, dtype, kv8, heads, dim, page, layers, what):
    rng = np.random.default_rng(dim + page)
    lengths = [1, page, page + 1, 0, 2 * page - 1, 3]
    c = lc.new_cache(dtype, kv8, 12, page, heads, dim, len(lengths) + 1, 4, layers)
    table = lc.hold(c, lengths, rng)
    layer = layers - 1
    order = [4, 0, 2, 5, 1]
    counts = [1] * 5 if what == "step" else [page + 3, 1, 0, 3, page]
    first = np.concatenate([[0], np.cumsum(counts)])
    R = int(first[-1])
    # (keys and values side by side in a wider buffer, at odd addresses; of many magnitudes, a head of zeros)
    both = torch.from_numpy(rng.standard_normal((R, 2 * heads * dim + 3)).astype(np.float32) * np.float32(10.0) ** rng.integers(-9, 9, (R, 1)).astype(np.float32)).to(lc.DTYPES[dtype])
    both[0, 1:1 + dim] = 0
    both = both.cuda()
    k, v = both[:, 1:1 + heads * dim], both[:, 2 + heads * dim:2 + 2 * heads * dim]
    before = held(c)
    rows = []
    for b, s in enumerate(order):
        for r in range(first[b], first[b + 1]):
            t = lengths[s] - (int(first[b + 1]) - r)
            if t >= 0:
                rows.append((s, t, k[r].reshape(heads, dim), v[r].reshape(heads, dim)))
    for again in range(2):
        mt.kv_write(ctx, c, k, v, seqs=ints(order), first_row=None if what == "step" else ints(first), max_new=max(counts), layer=layer)
    same(held(c), written(before, c, table, dtype, kv8, rows, layer))


@pytest.mark.parametrize("dtype,kv8", KINDS)
def test_rows_without_a_place(ctx, dtype, kv8):
    """Numbers out of range, pages out of range, tokens beyond the table, rows in no sequence, rows outside: nothing is written for them."""
    rng = np.random.default_rng(3)
    heads, dim, page = 2, 32, 16
    lengths = [5, 40, 20, 33]
    c = lc.new_cache(dtype, kv8, 10, page, heads, dim, 4, 3)
    table = lc.hold(c, lengths, rng)
    bad = torch.from_numpy(table.copy())
    bad[1, 2], bad[2, 1] = 10, -5
    c.table.copy_(bad)
    c.lengths[3] = 60                              # (the table ends at 48)
    order = [-1, 1, 0, 4, 2, 3, 0x7fffffff]
    first = [2, 3, 13, 14, 15, 19, 34, 90]
    R = 36
    k, v = (torch.from_numpy(rng.standard_normal((R, heads * dim), dtype=np.float32)).to(lc.DTYPES[dtype]).cuda() for _ in range(2))
    before, rows = held(c), []
    for b, s in enumerate(order):
        for r in range(first[b], min(first[b + 1], R)):
            if 0 <= s < 4:
                t = [5, 40, 20, 60][s] - (first[b + 1] - r)
                if 0 <= t < 48 and 0 <= bad[s, t // page] < 10:
                    rows.append((s, t, k[r].reshape(heads, dim), v[r].reshape(heads, dim)))
    assert 3 < len(rows) < 25
    for max_new in (1, 5, 100):                    # (more rows than announced are written too)
        mt.kv_write(ctx, c, k, v, seqs=ints(order), first_row=ints(first), max_new=max_new)
        same(held(c), written(before, c, table, dtype, kv8, rows, 0))
    mt.kv_write(ctx, c, k[:0], v[:0], seqs=ints([]))
    mt.kv_write(ctx, c, k[:0], v[:0], seqs=ints([1]), first_row=ints([0, 0]))
    same(held(c), written(before, c, table, dtype, kv8, rows, 0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_values_in_8_bits(ctx, dtype):
    """Ties, the ends of the range, values below the smallest scale, infinities and NaN."""
    x = np.zeros((12, 64), dtype=np.float32)
    x[0, :8] = [448, 432, 416.5, 17, 19, -1.0625, 2.0 ** -9, 3 * 2.0 ** -10]        # (a scale of 1: ties to even)
    x[1, :4] = [448.0625 if dtype == "f32" else 450, 1, -3, 0.1]
    x[2, :3] = [2.0 ** 127, -2.0 ** 120, 1.5]
    x[3, :3] = [2.0 ** -126, 2.0 ** -127, -2.0 ** -130]
    x[4, :2] = [2.0 ** -133, -2.0 ** -133]
    x[5, 3], x[5, 4] = np.inf, 1
    x[6, 60], x[6, 4] = -np.inf, 1
    x[7, 63], x[7, 4] = np.nan, 1
    x[8] = -0.0
    x[9, :64] = np.arange(64) * 7.0
    x[10, :64] = 2.0 ** (np.arange(64) - 40.0)
    x[11, 5] = -2.0 ** -100
    c = lc.new_cache(dtype, True, 1, 16, 1, 64, 1, 1)
    c.table.zero_(), c.lengths.fill_(12)
    rows = torch.from_numpy(x).to(lc.DTYPES[dtype]).cuda()
    mt.kv_write(ctx, c, rows, rows, first_row=ints([0, 12]), max_new=12)
    finite = [i for i in range(12) if i not in (5, 6, 7)]
    want, e = lc.in_8_bits(lc.in_64(rows[finite]))
    for q, s in ((c.k.view(torch.uint8)[0, 0, 0, :12], c.k_scales), (c.v.view(torch.uint8)[0, 0, 0, :, :12].t(), c.v_scales)):
        q, s = q.cpu().numpy(), s.view(torch.uint8)[0, 0, 0, :12].cpu().numpy()
        assert np.array_equal(s[finite], e) and np.array_equal(q[finite], want)
        assert np.all(s[[5, 6, 7]] == 255) and np.all(q[[5, 6, 7]] & 127 == 127)


def test_captured_and_on_another_stream(ctx):
    rng = np.random.default_rng(5)
    heads, dim, page = 2, 64, 32
    c = lc.new_cache("bf16", True, 4, page, heads, dim, 2, 2, fill=0.0)
    table = lc.hold(c, [40, 33], rng)
    k, v = (torch.zeros(2, heads * dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    mt.kv_write(ctx, c, k, v)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mt.kv_write(ctx, c, k, v)
    for again in range(4):
        k.copy_(torch.from_numpy(rng.standard_normal((2, heads * dim))))
        v.copy_(torch.from_numpy(rng.standard_normal((2, heads * dim))))
        if again < 3:
            c.lengths.copy_(ints([40 - again, 33 - again]))
        torch.cuda.synchronize()
        before = held(c)
        lengths = c.lengths.tolist()
        if again % 2:
            mt.kv_write(ctx, c, k, v, stream=side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        same(held(c), written(before, c, table, "bf16", True, [(s, lengths[s] - 1, k[s].reshape(heads, dim), v[s].reshape(heads, dim)) for s in range(2)], 0))


def test_written_caches_count_as_changed(ctx):
    c = lc.new_cache("f32", False, 2, 16, 1, 16, 1, 2)
    c.table.copy_(ints([0, 1]).view(1, 2)), c.lengths.fill_(20)
    w = torch.ones_like(c.k, requires_grad=True)
    loss = (w * c.k).sum()
    x = torch.zeros(1, 16, device="cuda")
    mt.kv_write(ctx, c, x, x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_places_far_into_a_large_cache(ctx):
    """Elements beyond 2^32."""
    page, heads, dim = 256, 4, 128
    stride = page * heads * dim
    pages = (1 << 32) // stride + 3
    c = mt.alloc_kv(pages, page, heads, dim, 2, 1, dtype=mt.MT_BF16)
    c.table.copy_(ints([pages - 1, 0]).view(2, 1)), c.lengths.copy_(ints([200, 100]))
    c.k[0, 0].zero_(), c.v[0, 0].zero_(), c.k[0, -1].zero_(), c.v[0, -1].zero_()
    x = torch.randn(2, heads * dim, device="cuda", dtype=torch.bfloat16)
    mt.kv_write(ctx, c, x, -x)
    for s, p, t in ((0, pages - 1, 199), (1, 0, 99)):
        assert torch.equal(c.k[0, p, :, t].reshape(-1), x[s]) and torch.equal(c.v[0, p, :, :, t].reshape(-1), -x[s])
        assert int(c.k[0, p].count_nonzero()) == int(x[s].count_nonzero()) == int(c.v[0, p].count_nonzero())
