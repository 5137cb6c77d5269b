"""Plain evaluations in 64 bits of the operators behind language models' answers, and inputs for their tests (numpy, no GPU)."""
import numpy as np

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6])


def e4m3(codes):
    """Values of e4m3 bytes."""
    c = np.asarray(codes, dtype=np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def e8m0(codes):
    c = np.asarray(codes, dtype=np.float64)
    return np.where(c == 255, np.nan, 2.0 ** (c - 127))


def spread(scales, width):
    """A scale for every column."""
    return np.repeat(scales, 32, axis=1)[:, :width]


def random_matrix(rng, n, k, lo=118, hi=124):
    """(codes, scales, values) of an n x k matrix of 4-bit weights."""
    c = rng.integers(0, 16, (n, k + k % 2), dtype=np.uint8)
    if k % 2:
        c[:, -1] = rng.integers(0, 16, n)            # the half byte behind an odd row is nobody's
    scales = rng.integers(lo, hi, (n, -(-k // 32)), dtype=np.uint8)
    return c[:, 0::2] | c[:, 1::2] << 4, scales, E2M1[c[:, :k]] * spread(e8m0(scales), k)


def scored(x, n_classes=None, allowed=None, given=None, top=0, temperature=1.0):
    """Everything mt_score returns for rows x (float64), and a bound for the entropies' and log probabilities' errors in fp32."""
    R, C = x.shape
    out = {"entropy": np.zeros(R), "given": None if given is None else np.full(given.shape, -np.inf), "ranks": None if given is None else np.full(given.shape, -1),
           "ids": np.full((R, top), -1), "top": np.full((R, top), -np.inf), "bound": np.zeros(R)}
    for r in range(R):
        n = C if n_classes is None else min(max(int(n_classes[r]), 0), C)
        ok = np.arange(C) < n
        if allowed is not None:
            ok &= (allowed[r][np.arange(C) // 32] >> (np.arange(C) % 32).astype(np.uint32)) & 1 == 1
        ok &= ~(x[r] == -np.inf)
        lost = bool(np.any(np.isnan(x[r][ok]) | (x[r][ok] == np.inf)))
        ids = np.nonzero(ok)[0]
        if lost:
            out["entropy"][r] = np.nan
            out["top"][r] = np.nan
        if len(ids) and not lost:
            z = (x[r][ids] - x[r][ids].max()) / temperature
            s = np.exp(z).sum()
            lp = z - np.log(s)
            p = np.exp(lp)
            out["entropy"][r] = -(p * lp)[p > 0].sum()
            # fp32: an exponent is off by 2^-23 of itself, so e^z by |z| 2^-23, and z e^z by z^2 2^-23; sums and logarithms by a few 2^-23
            out["bound"][r] = 2.0 ** -21 * (1 + (p * z * z)[p > 0].sum() + out["entropy"][r])
            order = ids[np.argsort(-x[r][ids], kind="stable")]
            out["ids"][r, :len(order[:top])] = order[:top]
            by_class = np.full(C, -np.inf)
            by_class[ids] = lp
            out["top"][r, :len(order[:top])] = by_class[order[:top]]
            place = np.full(C, -1)
            place[order] = np.arange(len(order))
        if given is not None:
            for g, c in enumerate(given[r]):
                if 0 <= c < C and ok[c]:
                    out["given"][r, g] = np.nan if lost else by_class[c]
                    out["ranks"][r, g] = -1 if lost else place[c]
    return out
