"""The calls on a cache's pages against books of whole numbers, one entry at a time."""
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


class Pair:
    """A cache and its books, called together and compared.  Every page's contents are its first owner's: random bytes."""

    def __init__(self, ctx, pages, page, seqs, width, kv8=False, heads=1, dim=16, layers=2):
        self.ctx, self.b = ctx, lc.Books(pages, page, seqs, width)
        self.c = lc.new_cache("bf16", kv8, pages, page, heads, dim, seqs, width, layers)
        self.parts = [x for x in (self.c.k, self.c.v, self.c.k_scales, self.c.v_scales) if x is not None]
        g = torch.Generator("cuda").manual_seed(pages)
        for x in self.parts:
            x.view(torch.uint8).copy_(torch.randint(0, 256, x.view(torch.uint8).shape, generator=g, dtype=torch.uint8, device="cuda"))
        self.original = [x.view(torch.uint8).clone() for x in self.parts]

    def grow(self, seqs, tokens, **kw):
        granted = torch.full((len(tokens),), 9, dtype=torch.int32, device="cuda")
        mt.kv_grow(self.ctx, self.c, ints(tokens), seqs=None if seqs is None else ints(seqs), granted=granted, **kw)
        assert granted.tolist() == self.b.grow(range(len(tokens)) if seqs is None else seqs, tokens)
        return self

    def fork(self, parents, children, **kw):
        granted = torch.full((len(parents),), 9, dtype=torch.int32, device="cuda")
        mt.kv_fork(self.ctx, self.c, ints(parents), ints(children), granted=granted, **kw)
        assert granted.tolist() == self.b.fork(parents, children)
        return self

    def free(self, seqs, **kw):
        mt.kv_free(self.ctx, self.c, ints(seqs), **kw)
        self.b.free(seqs)
        return self

    def compact(self, **kw):
        live = ints([-1])
        mt.kv_compact(self.ctx, self.c, live=live, **kw)
        assert live.item() == self.b.compact()
        return self

    def check(self):
        b, c = self.b, self.c
        table = np.full(c.table.shape, -1, np.int32)
        for s, t in enumerate(b.table):
            table[s, :len(t)] = t
        assert c.lengths.tolist() == b.lengths
        assert c.refs.tolist() == b.refs
        assert np.array_equal(np.where(np.arange(table.shape[1]) < np.array([len(t) for t in b.table])[:, None], c.table.cpu().numpy(), -1), table)
        held = [p for p, r in enumerate(b.refs) if r > 0]
        if held:
            at, of = torch.tensor(held).cuda(), torch.tensor([b.contents[p] for p in held]).cuda()
            for x, o in zip(self.parts, self.original):
                assert torch.equal(x.view(torch.uint8)[:, at], o[:, of])
        return self


def test_growing(ctx):
    p = Pair(ctx, 40, 16, 6, 8)
    p.grow(None, [0, 1, 16, 17, 100, 5]).check()
    p.grow([3, 0, 5], [14, 0, 12]).check().grow([3], [1]).check()
    p.grow([0, 1, 4], [-1, 128, 28]).check()                     # negative; beyond the table's width; to its end
    p.grow([2, 2, 9, -1, 0], [3, 50, 5, 5, 1]).check()           # twice, and no sequences
    p.grow([1, 2, 3, 0], [127, 100, 60, 14]).check()             # more than there is: who comes late gets none, who needs none is served
    p.grow([], []).check()


def test_forks(ctx):
    p = Pair(ctx, 30, 16, 12, 6)
    p.grow([0, 1, 2, 3], [40, 32, 1, 0]).check()
    p.fork([0, 0, 1, 2, 3], [4, 5, 6, 7, 8]).check()
    p.grow([0, 4, 5, 6, 8], [8, 9, 30, 1, 3]).check()
    p.fork([4, 0, 0, 99, 1, 9, 3], [9, 9, 1, 10, -7, 10, 11]).check()       # a child twice, one that holds tokens, numbers of nobody, an empty parent
    p.free([0, 4]).check().fork([5, 5], [0, 4]).check()
    q = Pair(ctx, 5, 16, 6, 3)
    q.grow([0, 1], [40, 16]).check().fork([0, 1, 0, 1], [2, 3, 4, 5]).check()       # one page is left


def test_a_child_that_is_also_a_parent(ctx):
    """Parents count as they were before the call."""
    p = Pair(ctx, 30, 16, 5, 4)
    p.grow([0], [20]).check().fork([0, 1, 2], [1, 2, 3]).check()
    assert p.b.lengths == [20, 20, 0, 0, 0]


def test_releases(ctx):
    p = Pair(ctx, 40, 16, 8, 8)
    p.grow(None, [100, 1, 16, 0, 33]).check()
    p.fork([0, 4], [5, 6]).check()
    p.free([0, 0, 3, 99, -1, 4]).check().free([5, 1, 2, 6]).check()
    assert not p.c.refs.any() and torch.all(p.c.table == -1)


@pytest.mark.parametrize("kv8", [False, True])
def test_compaction(ctx, kv8):
    p = Pair(ctx, 50, 32, 10, 8, kv8, heads=3, dim=48)
    p.compact().check()
    p.grow(None, [200, 3, 100, 64, 33, 128, 5]).check().compact().check()
    p.fork([0, 2], [7, 8]).check().free([0, 1, 3]).check().compact().check()
    p.grow([1, 3], [150, 20]).check().free([2, 7]).compact().check().compact().check()
    p.free(range(10)).compact().check()


@pytest.mark.parametrize("pages,page,seqs,width,kv8", [(64, 16, 7, 20, True), (1000, 16, 90, 40, False), (40000, 16, 1500, 30, False)])
def test_random_lives(ctx, pages, page, seqs, width, kv8):
    rng = np.random.default_rng(pages)
    p = Pair(ctx, pages, page, seqs, width, kv8, layers=1)
    pick = lambda: rng.integers(-1, seqs + 1, rng.integers(1, seqs + 1)).tolist()  # noqa: E731
    for step in range(25 if pages < 10000 else 8):
        what = rng.integers(0, 7)
        if what <= 2:
            s = pick()
            p.grow(s, rng.integers(0, rng.choice([2, page, 3 * page]), len(s)).tolist())
        elif what == 3:
            s = pick()
            p.fork(s, rng.permutation(pick() + s)[:len(s)].tolist())
        elif what == 4:
            p.free(pick()[:max(1, seqs // 3)])
        else:
            p.compact()
        p.check()


@pytest.mark.parametrize("kv8", [False, True])
def test_copies(ctx, kv8):
    p = Pair(ctx, 20, 64, 2, 4, kv8, heads=2, dim=80, layers=3)
    before = [x.clone() for x in p.original]
    src, dst = [3, 4, 4, 20, 5, -1, 7, 8, 6], [10, 11, 12, 0, 20, 1, 7, 13, 13]          # out of range, onto itself, one target twice (the last counts)
    mt.kv_copy(ctx, p.c, ints(src), ints(dst))
    for x, b in zip(p.parts, before):
        for s, d in ((3, 10), (4, 11), (4, 12), (6, 13)):
            b[:, d] = b[:, s].clone()
        assert torch.equal(x.view(torch.uint8), b)
    mt.kv_copy(ctx, p.c, ints([]), ints([]))
    many = torch.arange(3000, dtype=torch.int32, device="cuda") % 9
    mt.kv_copy(ctx, p.c, many, many + 9)
    for x, b in zip(p.parts, before):
        b[:, 9:18] = b[:, :9].clone()
        assert torch.equal(x.view(torch.uint8), b)


def test_strides_and_captured(ctx):
    """Layers inside of pages, a table of a wider buffer; calls replayed as a graph on changing books."""
    p = Pair(ctx, 60, 16, 9, 5, True, heads=2, dim=32, layers=3)
    inside = lambda t: t.view(torch.uint8).transpose(0, 1).contiguous().view(t.dtype).transpose(0, 1)  # noqa: E731
    o = p.c
    wide = torch.full((9, 8), -1, dtype=torch.int32, device="cuda")
    p.c = mt.KVCache(inside(o.k), inside(o.v), inside(o.k_scales), inside(o.v_scales), wide[:, 1:6], o.lengths, o.refs, o.work, o.spec.dtype)
    p.parts = [p.c.k, p.c.v, p.c.k_scales, p.c.v_scales]
    a, b, n, granted = ints([0, 1, 2]), ints([5, 6, 7]), ints([1, 40, 17]), ints([0, 0, 0])

    def step():
        mt.kv_free(ctx, p.c, b)
        mt.kv_grow(ctx, p.c, n, seqs=a, granted=granted)
        mt.kv_fork(ctx, p.c, a, b)
        mt.kv_compact(ctx, p.c)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for again in range(5):
        graph.replay()
        p.b.free([5, 6, 7])
        assert granted.tolist() == p.b.grow([0, 1, 2], n.tolist())
        p.b.fork([0, 1, 2], [5, 6, 7])
        p.b.compact()
        p.check()
        n.copy_(ints([again, 10 + again, 3]))
        p.free([again % 3]).check()
    assert torch.all(wide[:, 0] == -1) and torch.all(wide[:, 6:] == -1)


def test_damaged_books_touch_nothing_outside(ctx):
    """Pages out of range in a table are passed over."""
    p = Pair(ctx, 10, 16, 3, 4)
    p.grow([0], [50])
    p.c.table[0, 1], p.c.table[0, 3] = 10, -3
    mt.kv_fork(ctx, p.c, ints([0]), ints([1]))
    assert p.c.table[1].tolist()[:3] == [0, 10, 2] and p.c.refs.tolist()[:4] == [2, 1, 2, 1] and int(p.c.refs.sum()) == 7
    mt.kv_free(ctx, p.c, ints([0, 1]))
    assert p.c.refs.tolist()[:3] == [0, 1, 0] and p.c.lengths.tolist() == [0, 0, 0]
    p.c.lengths[2] = 1000                                # (more than its table holds)
    mt.kv_fork(ctx, p.c, ints([2]), ints([1]))
    mt.kv_compact(ctx, p.c)
    mt.kv_free(ctx, p.c, ints([2]))
    assert p.c.lengths.tolist() == [0, 0, 0]


def test_many_pages(ctx):
    """More than one sweep of counts, free pages far behind."""
    pages = 300000
    c = mt.alloc_kv(pages, 16, 1, 16, 3, 10, dtype=mt.MT_BF16)
    c.refs.fill_(1)
    free = [17, 16384, 16399, 40000, 299999]
    c.refs[torch.tensor(free).cuda()] = 0
    granted = ints([0, 0])
    mt.kv_grow(ctx, c, ints([60, 32]), seqs=ints([1, 0]), granted=granted)
    assert granted.tolist() == [1, 0] and c.table[1, :4].tolist() == free[:4] and c.lengths.tolist() == [0, 60, 0] and int((c.refs == 0).sum()) == 1
    live = ints([0])
    c.k.zero_()
    c.k[0, 40000] = 5.0
    mt.kv_free(ctx, c, ints([1]))
    mt.kv_grow(ctx, c, ints([16 * 5]), seqs=ints([2]))
    mt.kv_compact(ctx, c, live=live)
    assert live.item() == pages and c.table[2, :5].tolist() == free
    c.refs.zero_()
    c.refs[torch.tensor(free).cuda()] = 1
    mt.kv_compact(ctx, c, live=live)
    assert live.item() == 5 and c.table[2, :5].tolist() == [0, 1, 2, 3, 4] and c.refs[:6].tolist() == [1, 1, 1, 1, 1, 0] and torch.all(c.k[0, 3] == 5.0) and int(c.refs.sum()) == 5


def test_calls_on_tensors_refuse(ctx):
    c = mt.alloc_kv(10, 16, 1, 16, 3, 4)
    for f, args in ((mt.kv_grow, (ints([1]).long(),)), (mt.kv_grow, (ints([1]), ints([1, 2]))), (mt.kv_grow, (ints([1]), None, ints([1, 2]))), (mt.kv_grow, (None,)), (mt.kv_fork, (ints([1]), ints([1, 2]))),
                    (mt.kv_fork, (None, ints([1]))), (mt.kv_free, (torch.zeros(1, dtype=torch.int32),)), (mt.kv_free, (None,)), (mt.kv_compact, (ints([1, 2]),)), (mt.kv_copy, (ints([1]), None)),
                    (mt.kv_copy, (ints([1, 2]), ints([1]))), (mt.kv_free, (ints([1]).view(1, 1),))):
        with pytest.raises(ValueError):
            f(ctx, c, *args)
    with pytest.raises(mt.MtError):
        mt.kv_free(ctx, c, ints([0, 1, 2, 0]))
    with pytest.raises(ValueError):
        mt.torch_io.answers().kv_free(ctx._h.value, 0, 0, None, c._tensors, ints([0]))
