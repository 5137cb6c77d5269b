"""mt_attend where sequences are cut into parts that the last of them joins."""
import numpy as np
import pytest
import torch

import lm_cache_common as lc
import paper_1901_06887_amd as mt
from test_gpu_lm_attend import KINDS, Case, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("length", [700, 1500, 4096, 5000])
@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinite_value_in_any_part(ctx, dtype, new, length, sign):
    """Infinite in its own element of the rows that see it, wherever its token stands; everything else is as it was."""
    for at in (0, 300, length // 2, length - 4, length - 1):
        c = Case(dtype, False, 2, 2, 64, 16, [length], new=[new])
        want = c.want()
        value = c.v[0][at:at + 1].copy()
        value[0, 1, 5] = sign * np.inf
        lc.put(c.c, c.table, 0, torch.from_numpy(c.k[0][at:at + 1]).to(lc.DTYPES[dtype]), torch.from_numpy(value).to(lc.DTYPES[dtype]), 0, at)
        out, lse = c.call(ctx)
        sees = np.array([length - (new - 1 - j) > at for j in range(new)])
        odd = np.zeros((new, 4, 64), dtype=bool)
        odd[sees, 2:, 5] = True
        got = lc.in_64(out).reshape(odd.shape)
        assert np.all(got[odd] == sign * np.inf), (at, got[odd])
        rest = [np.where(odd, 0.0, w.reshape(odd.shape)).reshape(new, -1) for w in (got, want[0], want[2])]
        c.check((torch.from_numpy(rest[0]), lse), (rest[1], want[1], rest[2], want[3]))


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("heads,group,dim,page,new", [(2, 5, 80, 32, [1, 5, 3, 4]), (1, 17, 64, 16, [2, 5, 0, 5]), (2, 4, 128, 64, [3, 16, 9, 1]), (1, 3, 256, 128, [2, 16, 1, 16]), (2, 17, 48, 16, [1, 1, 1, 1]), (1, 40, 128, 32, [3, 2, 1, 3])])
@pytest.mark.parametrize("window", [0, 600, 1000, 2600])
def test_parts_of_several_tiles(ctx, dtype, kv8, heads, group, dim, page, new, window):
    """Several new tokens and more query heads than a tile has columns, over sequences of one part and of many; windows whose rows begin in different parts."""
    c = Case(dtype, kv8, heads, group, dim, page, [3, 700, 1531, 5000], new=new, peak=2.0)
    assert mt.attend_scratch(c.c.spec, 4, c.q_heads, max(new), 5000) > 0
    want = c.want(window)
    got = c.call(ctx, window=window)
    c.check(got, want)
    again = c.call(ctx, window=window)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("heads,group,dim,length", [(1, 4, 64, 1500), (2, 17, 80, 1029), (1, 5, 128, 770), (1, 2, 256, 4097)])
def test_odd_values_that_some_rows_see_in_the_last_part(ctx, dtype, kv8, heads, group, dim, length):
    """NaN and infinities among the new tokens, at the borders of parts, and in front of the window: rows that do not see them are finite, those that do are not."""
    odd = lambda x: (np.full((1, heads, dim), x, np.uint8), np.full((1, heads), 255, np.uint8)) if kv8 else torch.full((1, heads, dim), float("nan") if x else float("inf"), dtype=lc.DTYPES[dtype])  # noqa: E731
    for window, tokens, bad in ((0, [length - 2], [3, 4]), (0, [length - 1], [4]), (0, [length - 4, length - 1], [1, 2, 3, 4]), (600, [length - 604], [0]), (600, [length - 602, length - 2], [0, 1, 2, 3, 4]),
                                (length - 1024, [length - 2], [3, 4])):
        c = Case(dtype, kv8, heads, group, dim, 32, [length, 40], new=[5, 2])
        want = c.want(window if window > 0 else 0)
        for i, t in enumerate(tokens):
            lc.put(c.c, c.table, 0, odd(0x7f if kv8 else i % 2), odd(0x30 if kv8 else 1), 0, t)
        out, lse = c.call(ctx, window=max(window, 0))
        good = [r for r in range(7) if r not in bad]
        assert torch.all(torch.isnan(out[bad])), (window, tokens)
        c.check((out[good], lse[good]), tuple(w[good] for w in want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_in_place_captured_and_with_many_tiles(ctx, dtype):
    """Outputs over the queries, in a graph that is replayed as sequences grow; a scratch that calls of other sizes have used."""
    c = Case(dtype, False, 2, 17, 64, 16, [3000, 900, 20], new=[4, 4, 4], width=200)
    scratch = mt.alloc_attend(ctx, c.c, c.q_heads, 3, 4, 3200)
    other = Case(dtype, False, 2, 17, 64, 16, [2000, 100, 20], new=[1, 1, 1], width=200)
    out, lse = torch.empty_like(c.q), torch.empty(12, c.q_heads, device="cuda")
    call = lambda: mt.attend(ctx, c.c, out, out, first_row=rows, max_new=4, max_length=3200, scale=c.scale, lse=lse,  # noqa: E731
                             scratch=scratch)
    rows = torch.tensor([0, 4, 8, 12], dtype=torch.int32, device="cuda")
    out.copy_(c.q)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for again in range(4):
        c.lengths = [3000 - 511 * again, 900 - 256 * again, 20 - 6 * again]
        c.c.lengths.copy_(torch.tensor(c.lengths, dtype=torch.int32))
        c.q.copy_(torch.randn_like(c.q))
        out.copy_(c.q)
        torch.cuda.synchronize()
        want = c.want()
        graph.replay()
        other.check(other.call(ctx, max_length=3200, scratch=scratch), other.want())
        torch.cuda.synchronize()
        c.check((out, lse), want)
