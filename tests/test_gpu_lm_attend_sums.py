"""mt_attend: what lse says about infinite products, and how far weights are off."""
import numpy as np
import pytest
import torch

import lm_cache_common as lc
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
