"""mt_attend against a plain evaluation in 64 bits.  Caches are NaN wherever no token stands."""
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


class Case:
    """A cache of sequences of the given lengths, and rows for the last new[b] tokens of sequence order[b]."""

    def __init__(self, dtype, kv8, heads, group, dim, page, lengths, new=None, order=None, layers=1, spare=2, seed=0, peak=1.0, width=None):
        rng = np.random.default_rng(seed + dim + page + sum(lengths))
        self.dtype, self.heads, self.q_heads, self.dim, self.lengths = dtype, heads, heads * group, dim, list(lengths)
        pages = sum(-(-n // page) for n in lengths) + spare
        width = width or max(1, max(-(-n // page) for n in lengths))
        self.layer = layers - 1
        self.c = lc.new_cache(dtype, kv8, pages, page, heads, dim, len(lengths), width, layers)
        self.table = lc.hold(self.c, lengths, rng, spare)
        self.k, self.v = [], []
        for s, n in enumerate(lengths):
            k, v = (lc.random_kv(rng, dtype, kv8, n, heads, dim) for _ in range(2))
            lc.put(self.c, self.table, s, k, v, self.layer)
            self.k.append(lc.values_of(k)), self.v.append(lc.values_of(v))
        self.order = list(range(len(lengths))) if order is None else order
        self.new = [1] * len(self.order) if new is None else new
        self.first = np.concatenate([[0], np.cumsum(self.new)])
        R = int(self.first[-1])
        self.scale = peak * dim ** -0.5 / (200.0 if kv8 else 1.0)             # (random bytes are of any magnitude up to 448)
        self.q = torch.from_numpy(rng.standard_normal((R, self.q_heads * dim), dtype=np.float32)).to(lc.DTYPES[dtype]).cuda()

    def want(self, window=0, reach=1 << 40):
        R = self.q.shape[0]
        out, lse, off, off_lse = np.zeros((R, self.q_heads, self.dim)), np.full((R, self.q_heads), -np.inf), np.zeros((R, self.q_heads, self.dim)), np.zeros((R, self.q_heads))
        q = lc.in_64(self.q).reshape(R, self.q_heads, self.dim)
        for b, s in enumerate(self.order):
            for r in range(self.first[b], self.first[b + 1]):
                if 0 <= s < len(self.lengths):
                    end = self.lengths[s] - (int(self.first[b + 1]) - r) + 1
                    begin = max(0, end - window) if window else 0
                    out[r], lse[r], off[r], off_lse[r] = lc.attended(q[r], self.k[s], self.v[s], begin, max(min(end, reach), 0), float(np.float32(self.scale)), self.dtype)
        return out.reshape(R, -1), lse, off.reshape(R, -1), off_lse

    def call(self, ctx, q=None, out=None, lse=True, max_new=None, max_length=None, scratch=None, **kw):
        q = self.q if q is None else q
        out = torch.full_like(self.q, float("nan")) if out is None else out
        lse = torch.full((self.q.shape[0], self.q_heads), float("nan"), device="cuda") if lse else None
        max_new = max(max(self.new), 1) if max_new is None else max_new
        max_length = max(self.lengths) if max_length is None else max_length
        if scratch is None:
            scratch = mt.alloc_attend(ctx, self.c, self.q_heads, len(self.order), max_new, max_length)
        plain = self.order == list(range(len(self.lengths)))
        mt.attend(ctx, self.c, q, out, seqs=None if plain else ints(self.order), first_row=None if self.new == [1] * len(self.order) else ints(self.first), max_new=max_new,
                  max_length=max_length, scale=self.scale, lse=lse, layer=self.layer, scratch=scratch, **kw)
        return out, lse

    def check(self, got, want):
        out, lse, off, off_lse = want
        o = lc.in_64(got[0])
        assert np.all(np.isfinite(o)) and np.all(np.abs(o - out) <= off), np.max((np.abs(o - out) - off) / (np.abs(out).max() + 1e-30))
        if got[1] is not None:
            n = lc.in_64(got[1])
            none = np.isneginf(lse)
            assert np.array_equal(np.isneginf(n), none)
            assert np.all(np.abs(n[~none] - lse[~none]) <= off_lse[~none])


KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("heads,group,dim,page", [(1, 1, 16, 16), (2, 4, 64, 16), (3, 5, 80, 32), (2, 8, 128, 64), (1, 16, 112, 128), (2, 17, 128, 16), (1, 2, 256, 256), (1, 40, 192, 32), (2, 3, 48, 64)])
def test_single_tokens(ctx, dtype, kv8, heads, group, dim, page):
    """Lengths of none, of one, around pages and tiles."""
    c = Case(dtype, kv8, heads, group, dim, page, [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, page, page + 1, 2 * page - 1, 300])
    c.check(c.call(ctx), c.want())


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("dim,page,lengths", [(64, 16, [5000]), (128, 64, [3001, 0, 17, 2048]), (128, 256, [20000]), (256, 32, [1, 4097])])
def test_long_caches(ctx, dtype, kv8, dim, page, lengths):
    """The cache is shared among workgroups."""
    c = Case(dtype, kv8, 2, 4, dim, page, lengths, peak=3.0)
    c.check(c.call(ctx), c.want())
    c.check(c.call(ctx, lse=False), c.want())
    c.check(c.call(ctx, max_length=0), c.want())


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("heads,group,dim,page,window", [(2, 2, 64, 16, 0), (1, 5, 80, 32, 40), (2, 4, 128, 64, 0), (1, 16, 128, 128, 1), (1, 20, 48, 16, 7), (1, 1, 256, 64, 33)])
def test_several_new_tokens(ctx, dtype, kv8, heads, group, dim, page, window):
    """Each up to itself; sequences in another order, one without rows, one of rows alone; windows."""
    c = Case(dtype, kv8, heads, group, dim, page, [70, 5, 33, 128, 1, 300], new=[3, 5, 0, 40, 17], order=[5, 1, 0, 3, 2])
    c.check(c.call(ctx, window=window), c.want(window))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 1000, 100000])
def test_windows(ctx, dtype, kv8, window):
    c = Case(dtype, kv8, 2, 4, 64, 32, [1, 63, 64, 66, 1500, 0])
    c.check(c.call(ctx, window=window), c.want(window))


@pytest.mark.parametrize("dtype,kv8", KINDS)
def test_announced_sizes_that_are_too_small(ctx, dtype, kv8):
    """More rows and longer sequences than announced are served too."""
    c = Case(dtype, kv8, 2, 3, 64, 16, [700, 4000, 60], new=[1, 70, 33])
    for max_new, max_length in ((1, 16), (2, 100), (70, 1), (1, 4000)):
        c.check(c.call(ctx, max_new=max_new, max_length=max_length), c.want())
    c.check(c.call(ctx, max_new=100000, max_length=1 << 31, scratch=torch.zeros(mt.attend_scratch(c.c.spec, 3, c.q_heads, 100000, 1 << 31), dtype=torch.uint8, device="cuda")), c.want())


@pytest.mark.parametrize("dtype,kv8", KINDS)
def test_rows_of_nobody(ctx, dtype, kv8):
    """Numbers out of range answer with 0; rows in no sequence, or outside of the call's, stay as they are; rows in front of a sequence's first token see nothing."""
    c = Case(dtype, kv8, 1, 2, 64, 16, [40, 3], new=[2, 1, 1, 6], order=[0, -1, 2, 1])
    R = c.q.shape[0]
    out = torch.full((R + 4, c.q.shape[1]), 7.0, dtype=c.q.dtype, device="cuda")
    lse = torch.full((R + 4, c.q_heads), 7.0, device="cuda")
    q = torch.cat([torch.full_like(out[:2], float("nan")), c.q, torch.full_like(out[:2], float("nan"))])
    mt.attend(ctx, c.c, q, out, seqs=ints(c.order), first_row=ints(c.first + 2), max_new=6, scale=c.scale, lse=lse, scratch=mt.alloc_attend(ctx, c.c, c.q_heads, 4, 6))
    c.check((out[2:-2], lse[2:-2]), c.want())
    for t in (out, lse):
        assert torch.all(t[:2] == 7) and torch.all(t[-2:] == 7)
    # row numbers outside of the call's rows
    out.fill_(7.0)
    mt.attend(ctx, c.c, q, out, seqs=ints([0, 1]), first_row=ints([-3, 2, 100]), max_new=6, scale=c.scale, scratch=mt.alloc_attend(ctx, c.c, c.q_heads, 2, 6))
    torch.cuda.synchronize()
    mt.attend(ctx, c.c, q[:0], out[:0], seqs=ints([]))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("max_new", [1, 3, 40])
def test_row_numbers_of_any_value(ctx, dtype, kv8, max_new):
    """No row is touched that first_row does not put inside of the call's rows; nor are pages, by a write."""
    c = Case(dtype, kv8, 1, 2, 64, 16, [40, 3])
    low, high = -2 ** 31, 2 ** 31 - 1
    for first in ([low, low], [high, high], [low, high], [high, low], [5, low], [low, -1], [3, 2], [7, 100], [-5, 0]):
        out = torch.full_like(c.q, 7.0)
        mt.attend(ctx, c.c, c.q, out, seqs=ints([0]), first_row=ints(first), max_new=max_new, scale=c.scale, scratch=mt.alloc_attend(ctx, c.c, c.q_heads, 1, max_new))
        touched = [r for r in range(2) if first[0] <= r < first[1]]
        assert torch.equal((out != 7.0).any(1).cpu(), torch.tensor([r in touched for r in range(2)]))
        if not touched or first[1] > 1000:
            before = [t.view(torch.uint8).clone() for t in (c.c.k, c.c.v)]
            mt.kv_write(ctx, c.c, c.q[:, :64], c.q[:, :64], seqs=ints([0]), first_row=ints(first), max_new=max_new)
            assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(before, (c.c.k, c.c.v)))


@pytest.mark.parametrize("dtype,kv8", KINDS)
def test_pages_out_of_range_are_not_seen(ctx, dtype, kv8):
    """... and tokens beyond the table."""
    c = Case(dtype, kv8, 2, 4, 64, 16, [100, 64])
    c.c.table[0, 2], c.c.table[0, 4], c.c.table[1, 3] = -1, c.c.k.shape[1], 0x7fffffff
    got = c.call(ctx)
    for s, gone in ((0, (2, 4)), (1, (3,))):
        there = np.array([t for t in range(c.lengths[s]) if t // 16 not in gone])
        c.k[s], c.v[s] = c.k[s][there], c.v[s][there]
        c.lengths[s] = len(there)
    c.check(got, c.want())
    c = Case(dtype, kv8, 1, 2, 64, 16, [48], new=[4])
    c.c.lengths.fill_(50)
    c.lengths = [50]
    c.check(c.call(ctx), c.want(reach=48))
    c.check(c.call(ctx, window=5), c.want(5, reach=48))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("new", [1, 3])
def test_strides_and_in_place(ctx, dtype, kv8, new):
    """Queries in a wider buffer at odd addresses; outputs over them; a cache whose layers lie inside of its pages."""
    c = Case(dtype, kv8, 2, 3, 80, 32, [333, 20, 64], new=[new] * 3, layers=2)
    want = c.want()
    wide = torch.zeros(c.q.shape[0], c.q.shape[1] + 7, dtype=c.q.dtype, device="cuda")
    q = wide[:, 3:3 + c.q.shape[1]]
    q.copy_(c.q)
    out = torch.full((c.q.shape[0], c.q.shape[1] + 3), 7.0, dtype=c.q.dtype, device="cuda")
    got = c.call(ctx, q=q, out=out[:, 1:-2])
    c.check(got, want)
    assert torch.all(out[:, :1] == 7) and torch.all(out[:, -2:] == 7)
    c.check(c.call(ctx, q=q, out=q), want)
    assert torch.all(wide[:, :3] == 0) and torch.all(wide[:, -4:] == 0)
    inside = lambda t: None if t is None else t.view(torch.uint8).transpose(0, 1).contiguous().view(t.dtype).transpose(0, 1)  # noqa: E731
    old = c.c
    c.c = mt.KVCache(inside(old.k), inside(old.v), inside(old.k_scales), inside(old.v_scales), old.table, old.lengths, old.refs, old.work, old.spec.dtype)
    assert c.c.k.stride(0) < c.c.k.stride(1)
    c.check(c.call(ctx), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 80])
def test_infinities_and_nan(ctx, dtype, dim):
    """A NaN, or a product of +infinity, makes its own rows NaN; products of -infinity weigh nothing, and a row of nothing else sees nothing."""
    H, page, lengths = 2, 16, [40, 40, 40, 40, 40, 40]
    c = Case(dtype, False, H, 2, dim, page, lengths)
    c.q.fill_(1.0)
    put = lambda s, t, h, k=None, v=None: lc.put(c.c, c.table, s, *(torch.from_numpy(x).to(lc.DTYPES[dtype]) for x in (kk(s, t, h, k), vv(s, t, h, v))), 0, t)  # noqa: E731

    def kk(s, t, h, x):
        if x is not None:
            c.k[s][t, h] = 0
            c.k[s][t, h, dim - 1] = x
        return c.k[s][t:t + 1]

    def vv(s, t, h, x):
        if x is not None:
            c.v[s][t, h, 3] = x
        return c.v[s][t:t + 1]

    put(0, 7, 0, k=np.nan)
    put(1, 39, 1, v=np.nan)
    put(2, 0, 0, k=np.inf)
    put(3, 20, 1, k=-np.inf)
    for t in range(40):
        put(4, t, 0, k=-np.inf)
    put(5, 11, 0, v=np.inf)
    out, lse = c.call(ctx)
    o, n = lc.in_64(out).reshape(6, H, 2, dim), lc.in_64(lse).reshape(6, H, 2)
    assert np.all(np.isnan(o[0, 0])) and np.all(np.isnan(n[0, 0])) and np.all(np.isfinite(o[0, 1]))
    assert np.all(np.isnan(o[1, 1, :, 3])) and np.all(np.isfinite(np.delete(o[1, 1], 3, -1))) and np.all(np.isfinite(n[1])) and np.all(np.isfinite(o[1, 0]))
    assert np.all(np.isnan(o[2, 0])) and np.all(np.isfinite(o[2, 1]))
    assert np.all(o[4, 0] == 0) and np.all(np.isneginf(n[4, 0])) and np.all(np.isfinite(o[4, 1]))
    assert np.all(np.isposinf(o[5, 0, :, 3])) and np.all(np.isfinite(np.delete(o[5, 0], 3, -1)))
    q = lc.in_64(c.q).reshape(6, 2 * H, dim)
    want = lc.attended(q[3], c.k[3], c.v[3], 0, 40, c.scale, dtype)
    assert np.all(np.abs(o[3].reshape(-1, dim) - want[0]) <= want[2])


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("window", [0, 6])
def test_odd_values_in_tokens_that_only_later_rows_see(ctx, dtype, kv8, window):
    """Tokens of NaN and infinity among the new ones, and in front of the window: rows that do not see them are finite."""
    c = Case(dtype, kv8, 1, 4, 64, 16, [50, 34], new=[5, 4])
    want = c.want(window)
    odd = lambda: (np.full((1, 1, 64), 0x7f, np.uint8), np.full((1, 1), 127, np.uint8)) if kv8 else torch.full((1, 1, 64), float("nan"), dtype=lc.DTYPES[dtype])  # noqa: E731
    inf = lambda: (np.full((1, 1, 64), 0x30, np.uint8), np.full((1, 1), 255, np.uint8)) if kv8 else torch.full((1, 1, 64), float("inf"), dtype=lc.DTYPES[dtype])  # noqa: E731
    lc.put(c.c, c.table, 0, odd(), odd(), 0, 48)         # seen by the rows of tokens 48 and 49
    lc.put(c.c, c.table, 1, inf(), odd(), 0, 33)         # ... of token 33
    bad = [3, 4, 8]
    if window:
        lc.put(c.c, c.table, 0, odd(), inf(), 0, 41)     # seen by the rows of tokens 45 and 46
        bad = [0, 1, 3, 4, 8]
    out, lse = c.call(ctx, window=window)
    good = [r for r in range(9) if r not in bad]
    assert torch.all(torch.isnan(out[bad])) and torch.all(torch.isnan(lse[bad]))
    c.check((out[good], lse[good]), tuple(w[good] for w in want))


def test_parts_of_a_cache_joined_by_their_lse(ctx):
    c = Case("f32", False, 2, 4, 64, 16, [600])
    whole = c.want()
    k, v, both = c.k[0], c.v[0], []
    for begin, end in ((0, 250), (250, 600)):
        part = Case("f32", False, 2, 4, 64, 16, [end - begin])
        lc.put(part.c, part.table, 0, torch.from_numpy(k[begin:end]).float(), torch.from_numpy(v[begin:end]).float())
        part.q.copy_(c.q)
        o, n = part.call(ctx)
        both.append((lc.in_64(o).reshape(8, 64), lc.in_64(n).reshape(8, 1)))
    total = np.logaddexp(both[0][1], both[1][1])
    joined = sum(o * np.exp(n - total) for o, n in both)
    assert np.all(np.abs(joined.reshape(1, -1) - whole[0]) <= 4 * whole[2])


def test_results_do_not_depend_on_timing(ctx):
    c = Case("bf16", True, 4, 8, 128, 32, [9000, 100, 4000], peak=2.0)
    first = c.call(ctx)
    for _ in range(5):
        again = c.call(ctx)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_captured_replayed_and_on_two_streams(ctx):
    """Two graphs and calls between them share one scratch, one after the other; another stream with another scratch runs beside them."""
    c = Case("bf16", False, 2, 8, 128, 64, [5000, 3000])
    scratch, other = (mt.alloc_attend(ctx, c.c, c.q_heads, 2, 1, 5000) for _ in range(2))
    outs = [torch.zeros_like(c.q) for _ in range(4)]
    call = lambda o, s, **kw: mt.attend(ctx, c.c, c.q, o, max_length=5000, scale=c.scale, scratch=s, **kw)  # noqa: E731
    call(outs[0], scratch)
    torch.cuda.synchronize()
    graphs = []
    for o in outs[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(o, scratch)
    side = torch.cuda.Stream()
    for again in range(4):
        c.q.copy_(torch.randn_like(c.q))
        c.lengths = [5000 - 977 * again, 3000 - 64 * again]
        c.c.lengths.copy_(ints(c.lengths))
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        want = c.want()
        graphs[0].replay()
        call(outs[3], other, stream=side)
        call(outs[2], scratch)
        graphs[1].replay()
        torch.cuda.synchronize()
        for o in outs:
            c.check((o, None), want)


def test_tokens_far_into_a_large_cache(ctx):
    """Elements beyond 2^32, with values that tell pages apart."""
    page, heads, dim = 256, 4, 128
    pages = (1 << 32) // (page * heads * dim) + 3
    c = mt.alloc_kv(pages, page, heads, dim, 1, 3, dtype=mt.MT_BF16)
    c.table.copy_(ints([pages - 1, 0, pages - 2]).view(1, 3)), c.lengths.fill_(2 * page + 10)
    for p in (0, pages - 1, pages - 2):
        c.k[0, p].fill_(float("nan")), c.v[0, p].fill_(float("nan"))
    k, v = (torch.randn(2 * page + 10, heads, dim).to(torch.bfloat16) for _ in range(2))
    table = c.table.cpu().numpy()
    lc.put(c, table, 0, k, v)
    q = torch.randn(1, 8 * dim, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    mt.attend(ctx, c, q, out, scratch=mt.alloc_attend(ctx, c, 8, 1))
    want = lc.attended(lc.in_64(q).reshape(8, dim), lc.in_64(k), lc.in_64(v), 0, 2 * page + 10, float(np.float32(dim ** -0.5)), "bf16")
    assert np.all(np.abs(lc.in_64(out).reshape(8, dim) - want[0]) <= want[2])


def test_calls_on_tensors_refuse(ctx):
    c = Case("bf16", False, 2, 4, 64, 16, [40, 20])
    good = dict(q=c.q, out=torch.empty_like(c.q), scratch=mt.alloc_attend(ctx, c.c, 8, 2))
    call = lambda **kw: mt.attend(ctx, c.c, **{**good, **kw})  # noqa: E731
    call()
    for kw in (dict(q=c.q[:, :-1]), dict(q=c.q.half()), dict(out=good["out"].float()), dict(out=good["out"][:1]), dict(q=c.q.t()), dict(seqs=ints([0])), dict(seqs=ints([0, 1]).long()),
               dict(first_row=ints([])), dict(first_row=ints([0, 1]), seqs=ints([0, 1])), dict(lse=torch.zeros(2, 7, device="cuda")), dict(layer=-1), dict(window=-1), dict(max_new=-1),
               dict(scale="x"), dict(scratch=torch.zeros(8, device="cuda")), dict(seqs=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(layer=1), dict(max_new=0), dict(scale=float("nan"))):
        with pytest.raises(mt.MtError):
            call(**kw)
