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
