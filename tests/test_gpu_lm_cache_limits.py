"""Calls on caches at the ends of what lengths and lists may hold."""
import pytest
import torch

import lm_cache_common as lc
import paper_1901_06887_amd as mt

pytestmark = pytest.mark.gpu

HIGH = 2 ** 31 - 1
KINDS = [("bf16", False), ("f32", False), ("bf16", True), ("f32", True)]


@pytest.fixture(scope="module")
def ctx():
    c = mt.Context(1, 1, 64, 1, 1 << 16, mt.MT_BF16, 0)
    yield c
    c.close()


def ints(v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,kv8", KINDS)
@pytest.mark.parametrize("max_new", [1, 16, 40, 5000])
def test_lengths_near_the_end_of_32_bits_write_nothing(ctx, dtype, kv8, max_new):
    """Tokens beyond the table's width have no place, however far beyond; a sequence beside them is written."""
    page, rows = 16, 40
    lengths = [HIGH, HIGH - 1, HIGH - 63, HIGH - 64, HIGH - 262143, 2 ** 30, 48 + rows, 40]
    c = lc.new_cache(dtype, kv8, 24, page, 2, 32, len(lengths), 3)
    c.table.copy_(torch.arange(24, dtype=torch.int32).view(8, 3)), c.lengths.copy_(ints(lengths))
    x = torch.ones(rows * len(lengths), 64, dtype=lc.DTYPES[dtype], device="cuda")
    before = [t.view(torch.uint8).clone() for t in (c.k, c.v)]
    mt.kv_write(ctx, c, x, x, first_row=ints(range(0, rows * len(lengths) + 1, rows)), max_new=max_new)
    for t, b in zip((c.k, c.v), before):
        assert torch.equal(t.view(torch.uint8)[:, :21], b[:, :21])
    assert torch.all(c.k[0, 21:23].float() != 0) and torch.all(c.k[0, 21:23].float() == c.k[0, 21:23].float()) and torch.all(c.v[0, 21:23].float() == c.v[0, 21:23].float())
