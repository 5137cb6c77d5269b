"""Plain evaluations in 64 bits of the calls on language models' caches, and inputs for their tests."""
import numpy as np
import torch

import lm_common as lm
import paper_1901_06887_amd as mt

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}            # half a step of a rounding, relative to the value


def in_64(t):
    return t.double().cpu().numpy()


def new_cache(dtype, kv8, pages, page, heads, dim, seqs, width, layers=1, fill=float("nan")):
    """A cache whose elements are all `fill`."""
    c = mt.alloc_kv(pages, page, heads, dim, seqs, width, dtype=mt.MT_KV8 if kv8 else mt.MT_BF16 if dtype == "bf16" else mt.MT_F32, layers=layers)
    for x in (c.k, c.v):
        x.view(torch.uint8).fill_(0x7f) if kv8 else x.fill_(fill)            # (0x7f: NaN in e4m3)
    if kv8:
        c.k_scales.view(torch.uint8).fill_(255), c.v_scales.view(torch.uint8).fill_(255)
    return c


def hold(c, lengths, rng, spare=0):
    """Gives the sequences pages of random numbers."""
    page, pages = c.k.shape[3], c.k.shape[1]
    order, at = rng.permutation(pages), 0
    table, refs = np.full(c.table.shape, -1, np.int32), np.zeros(pages, np.int32)
    for s, n in enumerate(lengths):
        m = -(-n // page)
        table[s, :m] = order[at:at + m]
        refs[order[at:at + m]] += 1
        at += m
    assert at + spare <= pages
    c.table.copy_(torch.from_numpy(table)), c.refs.copy_(torch.from_numpy(refs)), c.lengths.copy_(torch.tensor([*lengths, *[0] * (len(table) - len(lengths))], dtype=torch.int32))
    return table


def put(c, table, s, k, v, layer=0, first=0):
    """Keys and values [tokens, heads, dim] (as the cache's type holds them) of sequence s from token `first` on; their values in 64 bits.  8 bits: bytes and e8m0 of [tokens, heads]."""
    page = c.k.shape[3]
    t = np.arange(first, first + len(k[0] if isinstance(k, tuple) else k))
    p, slot = torch.from_numpy(table[s, t // page].astype(np.int64)).cuda(), torch.from_numpy(t % page).cuda()
    for x, to, scales, turned in ((k, c.k, c.k_scales, False), (v, c.v, c.v_scales, True)):
        to = to[layer]
        if isinstance(x, tuple):
            x, e = x
            to = to.view(torch.uint8)
            scales[layer].view(torch.uint8)[p, :, slot] = torch.from_numpy(e).cuda()
        x = x if isinstance(x, torch.Tensor) else torch.from_numpy(x)
        if turned:
            to[p, :, :, slot] = x.cuda()
        else:
            to[p, :, slot] = x.cuda()


def values_of(x):
    return lm.e4m3(x[0]) * lm.e8m0(x[1])[..., None] if isinstance(x, tuple) else in_64(x)


def random_kv(rng, dtype, kv8, tokens, heads, dim):
    """Keys (or values) of so many tokens, as a cache holds them."""
    if kv8:
        return rng.integers(0, 256, (tokens, heads, dim), dtype=np.uint8) & 0xf7, rng.integers(118, 124, (tokens, heads), dtype=np.uint8)       # (no NaN)
    return torch.from_numpy(rng.standard_normal((tokens, heads, dim), dtype=np.float32)).to(DTYPES[dtype])


def attended(q, k, v, begin, end, scale, dtype):
    """out, lse and bounds for their errors, of one row q [q_heads, dim] over tokens begin .. end - 1 of k, v [tokens, heads, dim], all in 64 bits."""
    H, (QH, D) = k.shape[1], q.shape
    out, lse, off, off_lse = np.zeros((QH, D)), np.full(QH, -np.inf), np.zeros((QH, D)), np.zeros(QH)
    n = end - begin
    if n <= 0:
        return out, lse, off, off_lse
    for h in range(QH):
        kh, vh = k[begin:end, h * H // QH], v[begin:end, h * H // QH]
        x, size = kh @ q[h] * scale, np.abs(kh) @ np.abs(q[h]) * abs(scale)
        m = x.max()
        if m == -np.inf:
            continue
        p = np.exp(x - m)
        total = p.sum()
        p /= total
        out[h], lse[h] = p @ vh, m + np.log(total)
        # products of D terms in fp32, each addition off by 2^-24 of the magnitudes; the exponent by 2^-23 of itself twice (scaled, then subtracted); sums of n terms the same way; a
        # weight rounded to bf16 by half its step; the rescaling of sums a few roundings for each of at most n steps, which n counts again
        e = size.max() * (D + 2) * 2.0 ** -24 + 2.0 ** -22 * (np.abs(x).max() + np.abs(x - m).max()) + (2 * n + 16) * 2.0 ** -24
        off[h] = (2 * e + (STEP["bf16"] if dtype == "bf16" else 0.0)) * (p @ np.abs(vh)) + STEP[dtype] * np.abs(out[h]) + 1e-30
        off_lse[h] = e + 2.0 ** -22 * (1 + abs(lse[h]))
    return out, lse, off, off_lse


def in_8_bits(x):
    """Bytes and e8m0 of rows [.., dim] in 64 bits, to the nearest value, ties to even."""
    most = np.abs(x).max(-1)
    e = np.where(most > 0, np.ceil(np.log2(np.where(most > 0, most, 1) / 448)), 0)
    e = np.where(most > 448 * 2.0 ** e, e + 1, e)            # (where the logarithm was rounded)
    e = np.where((most <= 448 * 2.0 ** (e - 1)) & (most > 0), e - 1, e).clip(-126, 127)
    codes = np.arange(127)
    steps = lm.e4m3(codes)
    y = np.abs(x) / 2.0 ** np.where(most > 0, e, 0)[..., None]
    at = np.searchsorted(steps, y).clip(0, 126)
    low = np.maximum(at - 1, 0)
    up, down = steps[at] - y, y - steps[low]
    pick = np.where((down < up) | ((down == up) & (low % 2 == 0)), low, at)
    return (pick | np.where(np.signbit(x), 128, 0)).astype(np.uint8), (np.where(most > 0, e, 0) + 127).astype(np.uint8)


def sampled(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, n=None, allowed=None, bits=None):
    """(class, log of its share, classes kept) of one row x in 64 bits (float32 settings as given)."""
    C = len(x)
    bits = 62 - int(np.ceil(np.log2(C))) if bits is None else bits
    ok = np.arange(C) < (C if n is None else min(max(int(n), 0), C))
    if allowed is not None:
        ok &= (allowed[np.arange(C) // 32] >> (np.arange(C) % 32).astype(np.uint32)) & 1 == 1
    ok &= ~(x == -np.inf)
    settings = [float(v) for v in (u, temperature, top_p, min_p)]
    if np.any(np.isnan(x[ok]) | (x[ok] == np.inf)) or np.any(np.isnan(settings)) or temperature < 0:
        return -1, np.nan, -1
    ids = np.nonzero(ok)[0]
    if not len(ids):
        return -1, -np.inf, 0
    order = ids[np.argsort(-x[ids], kind="stable")]
    greedy = temperature < 2.0 ** -126
    with np.errstate(over="ignore"):
        z = (x[order] - x[order[0]]) / (1.0 if greedy else float(temperature)) if temperature < np.inf else np.zeros(len(order))
    w = np.exp(z)
    whole = [int(v) for v in np.rint(w * 2.0 ** bits)]
    keep = 1 if greedy else len(order) if top_k <= 0 else min(int(top_k), len(order))
    if min_p > 0:
        keep = min(keep, int((w >= min(float(min_p), 1.0)).sum()))
    if top_p < 1:
        target, total, m = max(1, int(np.ceil(max(float(top_p), 0.0) * float(sum(whole[:keep]))))), 0, 0
        while m < keep and total < target:
            total += whole[m]
            m += 1
        keep = m
    by_class = sorted((int(c), w) for c, w in zip(order[:keep], whole[:keep]))
    total = sum(w for _, w in by_class)
    at = float(u) * float(total)
    target = 0 if at <= 0 else total if at >= total else int(at)
    so_far, pick = 0, max(c for c, w in by_class if w)
    for c, w in by_class:
        so_far += w
        if so_far > target:
            pick = c
            break
    return pick, (x[pick] - x[order[0]]) / (1.0 if greedy else float(temperature)) - np.log(total / 2.0 ** bits), keep


class Books:
    """Tables, lengths and counts of a cache as whole numbers, with the calls on pages one entry at a time.  contents[p]: what stands in page p."""

    def __init__(self, pages, page, seqs, width):
        self.page, self.width = page, width
        self.refs, self.lengths, self.table = [0] * pages, [0] * seqs, [[] for _ in range(seqs)]
        self.contents = list(range(pages))

    def _free(self, n):
        found = [p for p, r in enumerate(self.refs) if r == 0]
        return found if n is None else found[:n]

    def grow(self, seqs, tokens):
        granted, named, pool, taken = [], set(), self._free(None), 0
        for s, t in zip(seqs, tokens):
            ok = 0 <= s < len(self.lengths) and s not in named and t >= 0
            named.add(s)
            if ok:
                need = -(-(self.lengths[s] + t) // self.page)
                take = need - len(self.table[s])
                ok = need <= self.width
                if ok:
                    taken += take
                    ok = take == 0 or taken <= len(pool)
                if ok:
                    for p in pool[taken - take:taken]:
                        self.refs[p] = 1
                        self.table[s].append(p)
                    self.lengths[s] += t
            granted.append(int(ok))
        return granted

    def fork(self, parents, children):
        granted, named, pool, taken, before = [], set(), self._free(None), 0, list(self.lengths)
        tables = [list(t) for t in self.table]
        moves = []
        for a, b in zip(parents, children):
            ok = 0 <= a < len(before) and 0 <= b < len(before) and b not in named and before[b] == 0
            named.add(b)
            if ok:
                part = before[a] % self.page != 0
                taken += part
                ok = not part or taken <= len(pool)
                if ok:
                    full = before[a] // self.page
                    self.table[b] = tables[a][:full]
                    for p in self.table[b]:
                        self.refs[p] += 1
                    if part:
                        p = pool[taken - 1]
                        self.table[b].append(p)
                        self.refs[p] = 1
                        moves.append((tables[a][full], p))
                    self.lengths[b] = before[a]
            granted.append(int(ok))
        for a, b in moves:
            self.contents[b] = self.contents[a]
        return granted

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lengths):
                for p in self.table[s]:
                    self.refs[p] -= 1
                self.table[s], self.lengths[s] = [], 0

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        src, dst = [p for p in range(live, len(self.refs)) if self.refs[p] > 0], [p for p in range(live) if self.refs[p] == 0]
        to = dict(zip(src, dst))
        for a, b in to.items():
            self.contents[b], self.refs[b], self.refs[a] = self.contents[a], self.refs[a], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return live
