"""What the bounds on attention's weights tell apart, on the oracle.  No GPU."""
import numpy as np
import pytest

import lm_cache_common as lc


def cut_off(p, bits):
    """p with its first so many bits."""
    m, e = np.frexp(p)
    return np.ldexp(np.floor(np.ldexp(m, bits)), e - bits)


def nearest(p, bits):
    m, e = np.frexp(p)
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def test_two_parts_of_a_weight():
    """The first eight bits, cut off, and eight of what is left: up to 2^-16 of the weight off, and not less everywhere."""
    p = np.random.default_rng(0).uniform(0, 256, 1 << 20).astype(np.float32).astype(np.float64)
    p = np.concatenate([p, 1 + 2.0 ** -8 + 2.0 ** -16 * np.linspace(0.9, 1.1, 999)])
    high = cut_off(p, 8)
    off = np.abs(high + nearest(p - high, 8) - p) / p
    assert 0.99 * 2.0 ** -16 < off.max() <= 2.0 ** -16


@pytest.mark.parametrize("n", [31, 300])
def test_a_missing_part_exceeds_the_bound(n):
    """Weights of the first eight bits alone, or with the rest of the token beside it, leave the bound that two parts keep."""
    rng = np.random.default_rng(n)
    k, v, q = rng.standard_normal((n, 1, 16)), rng.standard_normal((n, 1, 16)), rng.standard_normal((4, 16))
    want, _, off, _ = lc.attended(q, k, v, 0, n, 0.75, "f32")
    off = off + 2.0 ** -16 * lc.attended(q, k, np.abs(v), 0, n, 0.75, "f32")[0] + lc.STEP["bf16"] * np.abs(want)
    x = q @ k[:, 0].T * 0.75
    p = np.exp(x - x.max(1, keepdims=True))
    high = cut_off(p, 8)
    for weights, fits in ((high + nearest(p - high, 8), True), (high, False), (high + np.roll(nearest(p - high, 8), 1, 1), False)):
        out = weights @ v[:, 0] / p.sum(1, keepdims=True)
        # (outputs rounded to bf16)
        assert np.all(np.abs(nearest(out, 8) - want) <= off) == fits
