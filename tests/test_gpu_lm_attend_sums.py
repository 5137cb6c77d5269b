"""mt_attend: what lse says about infinite products, and how far weights are off."""
import numpy as np
import pytest
import torch

import lm_cache_common as lc
import lm_common as lm
import paper_1901_06887_amd as mt
from test_gpu_lm_attend import Case, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("length", [40, 1500])
def test_lse_of_infinite_products(ctx, dtype, new, length):
    """+infinity with a product of +infinity, whatever finite ones or -infinity stand beside it; NaN with a NaN among them, in any order; the row is NaN in either case, other heads and sequences are not."""
    inf, nan = np.inf, np.nan
    odd = [{0: inf}, {length - 3: inf}, {7: inf, length // 2: inf, length - 4: -inf}, {3: nan, 30: inf}, {3: inf, 30: nan}, {9: inf, 10: nan}, {length - 4: nan, 1: inf}, {5: -inf}]
    c = Case(dtype, False, 2, 2, 64, 16, [length] * len(odd), new=[new] * len(odd))
    c.q.fill_(1.0)
    for s, tokens in enumerate(odd):
        for t, x in tokens.items():
            c.k[s][t, 1] = 0
            c.k[s][t, 1, 9] = x
            lc.put(c.c, c.table, s, *(torch.from_numpy(y[s][t:t + 1]).to(lc.DTYPES[dtype]) for y in (c.k, c.v)), 0, t)
    out, lse = c.call(ctx)
    o, n = lc.in_64(out).reshape(len(odd), new, 4, 64), lc.in_64(lse).reshape(len(odd), new, 4)
    assert np.all(np.isfinite(o[:, :, :2])) and np.all(np.isfinite(n[:, :, :2]))
    for s, tokens in enumerate(odd):
        for j in range(new):
            seen = [x for t, x in tokens.items() if t <= length - new + j]
            if any(np.isnan(seen)):
                assert np.all(np.isnan(n[s, j, 2:])) and np.all(np.isnan(o[s, j, 2:])), (s, j, n[s, j])
            elif inf in seen:
                assert np.all(np.isposinf(n[s, j, 2:])) and np.all(np.isnan(o[s, j, 2:])), (s, j, n[s, j])
            else:
                assert np.all(np.isfinite(n[s, j, 2:])) and np.all(np.isfinite(o[s, j, 2:])), (s, j)


# A weight of bf16 rows is its first eight bits, cut off, and what is left (less than 2^-7 of the power of two below the weight), rounded to eight bits: off by up to 2^-16 of that power of two, half a step of
# values of 2^-8 to 2^-7 of it.
WEIGHT = 2.0 ** -16


class Close(Case):
    """Bounds with nothing of a weight's but WEIGHT where rows are bf16."""

    def want(self, window=0, reach=1 << 40):
        out, lse, off, off_lse = super().want(window, reach)
        if self.dtype == "bf16":
            # (sums and exponents as in fp32 rows, where weights are not rounded)
            self.dtype, signs = "f32", self.v
            off = super().want(window, reach)[2]
            self.v = [np.abs(v) for v in signs]
            off = off + WEIGHT * super().want(window, reach)[0] + lc.STEP["bf16"] * np.abs(out)
            self.dtype, self.v = "bf16", signs
        return out, lse, off, off_lse


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("heads,group,dim,page,lengths,new,peak", [(2, 4, 16, 16, [1, 2, 7, 16, 31, 33], [1] * 6, 3.0), (1, 17, 64, 32, [300, 40], [1, 1], 6.0), (2, 4, 128, 64, [5000, 700], [1, 1], 8.0),
                                                                   (2, 3, 64, 16, [9, 30, 200], [3, 1, 5], 4.0), (1, 8, 256, 128, [70, 1500], [2, 16], 8.0)])
def test_weights_in_two_parts(ctx, kv8, heads, group, dim, page, lengths, new, peak):
    c = Close("bf16", kv8, heads, group, dim, page, lengths, new=new, peak=peak)
    c.check(c.call(ctx), c.want())


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("new", [1, 2])
def test_weights_at_their_worst(ctx, kv8, new):
    """Weights of just over a half whose rest lies next to the middle of two values of eight bits, half of them below and with values of 1, half above and with -1: all of what is lost adds up, and little else is left."""
    n, dim = 14 + new, 16
    c = Case("bf16", kv8, 1, 1, dim, 16, [n], new=[new])
    c.scale = 1.0
    near = 0.5 + 2.0 ** -9 + 2.0 ** -17 * np.where(np.arange(n) % 2 == 0, 0.9, 1.1)
    near[0], near[15:] = 1.0, 1.0
    # the wanted products, as sums of parts that the cache's type holds, times powers of two
    factors = np.ones(dim) if not kv8 else 2.0 ** (-4.0 * np.minimum(np.arange(dim), 7))
    k, rest = np.zeros((n, 1, dim)), np.log(near)
    steps = np.sort(np.concatenate([s * lm.e4m3(np.arange(127)) for s in (1, -1)]))
    for d in range(8 if kv8 else 3):
        part = steps[np.abs(steps - (rest / factors[d])[:, None]).argmin(1)] if kv8 else lc.in_64(torch.from_numpy(rest / factors[d]).to(torch.bfloat16))
        k[:, 0, d], rest = part, rest - part * factors[d]
    assert np.all(np.abs(rest) < 2.0 ** -24)
    v = np.broadcast_to(np.where(np.arange(n) % 2 == 0, 1.0, -1.0)[:, None, None], k.shape).copy()
    v[0], v[15:] = 0, 0
    code = {float(x): i for i, x in reversed(list(enumerate(lm.e4m3(np.arange(256))))) if i & 127 != 127}
    hold = lambda x: (np.vectorize(code.get)(x).astype(np.uint8), np.full((n, 1), 127, np.uint8)) if kv8 else torch.from_numpy(x).to(torch.bfloat16)  # noqa: E731
    lc.put(c.c, c.table, 0, hold(k), hold(v))
    c.q.copy_(torch.from_numpy(np.tile(factors, (new, 1))))
    assert np.array_equal(lc.in_64(c.q), np.tile(factors, (new, 1))) and np.array_equal(lc.values_of(hold(k)), k)
    out = lc.in_64(c.call(ctx)[0])
    for j in range(new):
        end = n - new + 1 + j
        p = np.exp(k[:end, 0] @ factors)
        want, size = p @ v[:end, 0] / p.sum(), p @ np.abs(v[:end, 0]) / p.sum()
        # a weight's exponent is a sum of at most 8 products that adds up to less than 0.7 (8 roundings), scaled (2) and 2^x of it 2^-23 off; O adds up two parts of at most 16 tokens
        off = (WEIGHT + (0.7 * 10 + 2 + 32) * 2.0 ** -24) * size + (lc.STEP["bf16"] + 2.0 ** -18) * np.abs(want)
        assert np.all(np.abs(out[j] - want) <= off), (out[j, 0], want[0], off[0], (np.abs(out[j] - want) / size).max() * 2 ** 16)
        assert np.all(np.abs(out[j] - want) > 2.0 ** -17 * size)         # (the bound is not loose)
