"""The last step of several tenants' language models, for all their rows at once: a hidden layer and the layer over the vocabulary in 4-bit weights, a
norm in front of each, and what the logits say about the tokens that came next.

    python examples/answers.py [--tenants 8] [--rows 4] [--width 1024] [--hidden 4096] [--vocabulary 32768] [--steps 200]

    h  = x + delta                    delta: what the layers before left to be added
    q  = norm(h) * gain               in 8 bits, every row with its tenant's gain
    d  = W2 gelu(W1 q + b1)           W1, W2: the row's tenant's, in 4 bits
    q  = norm(h + d) * gain           in 8 bits
    l  = W3 q                         logits; a tenant's vocabulary may be shorter than the longest
    log p and rank of the next token, entropy, the five best tokens, of softmax(l / temperature)

Six launches, captured once as a graph and replayed for every step.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_1901_06887_amd as mt  # noqa: E402

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float32)


def to_4_bits(w):
    """Packed e2m1 codes (the even column in the low half) and e8m0 scales of fp32 weights [n, k]: every 32 along k share the least power of two
    at which none exceeds 6, each is the nearest value."""
    n, k = w.shape
    b = np.zeros((n, -(-k // 32) * 32), dtype=np.float32)
    b[:, :k] = w
    b = b.reshape(n, -1, 32)
    most = np.abs(b).max(2)
    e = np.where(most > 0, np.ceil(np.log2(np.maximum(most, 1e-30) / 6)), 0).clip(-100, 100)
    s = (b * np.exp2(-e)[:, :, None]).reshape(n, -1)[:, :k + k % 2]
    codes = np.searchsorted((E2M1[1:] + E2M1[:-1]) / 2, np.abs(s)).astype(np.uint8) | (s < 0).astype(np.uint8) << 3
    return codes[:, 0::2] | codes[:, 1::2] << 4, (e + 127).astype(np.uint8)


class AnswerStep:
    """Buffers and launches of the step for rows_of[t] rows of every tenant t.

    layers[t]: fp32 (W1 [hidden, width], b1 [hidden], W2 [width, hidden], W3 [vocabulary of t, width]); gains[t]: [width]."""

    def __init__(self, layers, gains, rows_of, top=5, temperature=1.0, device="cuda:0"):
        width, hidden = layers[0][0].shape[1], layers[0][0].shape[0]
        words = [w3.shape[0] for _, _, _, w3 in layers]
        need = sum(mt.matrix4_footprint(hidden, width) + mt.matrix4_footprint(width, hidden) + mt.matrix4_footprint(n, width) for n in words)
        self.ctx = mt.Context(1, 1, 64, 1, need + (1 << 20), mt.MT_BF16, torch.device(device).index or 0)
        first = np.concatenate([[0], np.cumsum(rows_of)])
        rows = int(first[-1])
        groups = []
        for pick in (0, 2, 3):
            numbers = []
            for one in layers:
                codes, scales = to_4_bits(one[pick])
                numbers.append(self.ctx.register_matrix4(*one[pick].shape, codes, scales, one[1] if pick == 0 else None))
            groups.append(mt.row_groups(zip(numbers, first, rows_of)))
        self.hidden_groups, self.back_groups, self.word_groups = groups
        tenant = np.repeat(np.arange(len(layers)), rows_of)
        buf = lambda n, dtype: torch.empty(rows, n, dtype=dtype, device=device)  # noqa: E731
        self.gain, self.tenant = torch.from_numpy(np.stack(gains)).to(device), torch.from_numpy(tenant.astype(np.int32)).to(device)
        self.n_words = torch.from_numpy(np.array(words, dtype=np.int32)[tenant]).to(device)
        # the step's inputs, to be written by the caller ...
        self.x, self.delta, self.next = buf(width, torch.bfloat16).zero_(), buf(width, torch.bfloat16).zero_(), buf(1, torch.int32).zero_()
        # ... what stands between its launches, and what it answers
        self.h, self.d, self.mid = buf(width, torch.bfloat16), buf(width, torch.bfloat16), buf(hidden, torch.bfloat16)
        self.q, self.q_scales = buf(width, torch.float8_e4m3fn), buf(-(-width // 32), torch.float8_e8m0fnu)
        self.q2, self.q2_scales = torch.empty_like(self.q), torch.empty_like(self.q_scales)
        self.logits = buf(max(words), torch.float32)
        self.scores = mt.alloc_scores(rows, 1, top, device=device)
        self.temperature, self.graph = temperature, None

    def launch(self, stream=None):
        """The six launches, on the given (or current) stream."""
        ctx, kw = self.ctx, dict(stream=stream)
        mt.add_norm(ctx, self.x, residual=self.delta, gain=self.gain, gain_ids=self.tenant, sum_out=self.h, out8=self.q, out8_scales=self.q_scales, **kw)
        mt.linear4(ctx, self.hidden_groups, self.q, self.mid, x_scales=self.q_scales, act=mt.MT_ACT_GELU, **kw)
        mt.linear4(ctx, self.back_groups, self.mid, self.d, **kw)
        mt.add_norm(ctx, self.h, residual=self.d, gain=self.gain, gain_ids=self.tenant, out8=self.q2, out8_scales=self.q2_scales, **kw)
        mt.linear4(ctx, self.word_groups, self.q2, self.logits, x_scales=self.q2_scales, **kw)
        return mt.score(ctx, self.logits, self.scores, given=self.next, n_classes=self.n_words, temperature=self.temperature, **kw)

    def run(self):
        """The same by replaying a graph; scores are ready when the current stream comes to what follows."""
        if self.graph is None:
            self.launch()
            torch.cuda.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.launch()
        self.graph.replay()
        return self.scores

    def close(self):
        self.graph = None
        self.ctx.close()


def random_tenants(rng, tenants, width, hidden, vocabulary):
    """Layers and gains; every other tenant's vocabulary is three quarters of the longest."""
    draw = lambda *shape: rng.standard_normal(shape, dtype=np.float32) * shape[-1] ** -0.5  # noqa: E731
    layers = [(draw(hidden, width), 0.1 * draw(hidden), draw(width, hidden), 4 * draw(vocabulary * 3 // 4 if t % 2 else vocabulary, width)) for t in range(tenants)]
    return layers, [1 + 0.1 * rng.standard_normal(width, dtype=np.float32) for _ in range(tenants)]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("tenants", 8), ("rows", 4), ("width", 1024), ("hidden", 4096), ("vocabulary", 32768), ("steps", 200)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args(argv)
    rng = np.random.default_rng(0)
    layers, gains = random_tenants(rng, a.tenants, a.width, a.hidden, a.vocabulary)
    step = AnswerStep(layers, gains, [a.rows] * a.tenants)
    rows = a.rows * a.tenants
    step.x.copy_(torch.from_numpy(rng.standard_normal((rows, a.width), dtype=np.float32)))
    step.delta.copy_(torch.from_numpy(0.3 * rng.standard_normal((rows, a.width), dtype=np.float32)))
    step.next.copy_(torch.from_numpy(rng.integers(0, a.vocabulary * 3 // 4, (rows, 1)).astype(np.int32)))
    for what, go in (("launches", step.launch), ("a graph", step.run)):
        o = go()
        torch.cuda.synchronize()
        start = time.perf_counter()
        for _ in range(a.steps):
            o = go()
        torch.cuda.synchronize()
        print("%d rows of %d tenants, as %s: %.1f us a step" % (rows, a.tenants, what, (time.perf_counter() - start) / a.steps * 1e6), flush=True)
    for r in range(0, rows, a.rows):
        print("tenant %d: log p %.3f, rank %d of the next token; entropy %.3f; best %s" %
              (r // a.rows, o.given_logprobs[r, 0], o.given_ranks[r, 0], o.entropy[r], o.top_ids[r].tolist()))
    step.close()


if __name__ == "__main__":
    main()
