"""Several tenants' language models answer prompts together: a paged cache that all of their sequences share, attention over it, and the choice of every next token.

    python examples/decode.py [--tenants 4] [--answers 2] [--prompt 200] [--tokens 32] [--layers 2] [--heads 8] [--kv_heads 2] [--head_dim 64] [--vocabulary 8192]

A layer adds Wo attend(q, cache) to the stream, with q, k, v = Wqkv (norm(x) * gain), Wqkv and Wo the row's tenant's in 4 bits; the last layer's stream gives, normed, the logits of the tenant's
vocabulary.  A prompt goes in whole, then becomes several answers that share its full pages and are drawn with settings of their own; every step makes room for a token, runs the
layers for all rows and draws.  The step is captured once and replayed; tables, lengths and free pages change on the device alone.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1901_06887_amd as mt  # noqa: E402
from answers import to_4_bits  # noqa: E402


def ints(values, device):
    return torch.tensor([int(v) for v in values], dtype=torch.int32, device=device)


class Rows:
    """Buffers of a pass over so many rows, those of tenant t side by side: rows_of[t]."""

    def __init__(self, models, rows_of):
        self.rows_of, rows, dev = list(rows_of), int(sum(rows_of)), models.device
        first = np.concatenate([[0], np.cumsum(rows_of)])
        buf = lambda n, dtype=torch.bfloat16: torch.empty(rows, n, dtype=dtype, device=dev)  # noqa: E731
        q, kv, w = models.q_width, models.kv_width, models.width
        self.groups = [[mt.row_groups(zip(layer[name], first, rows_of)) for name in ("qkv", "out")] for layer in models.layers]
        self.word_groups = mt.row_groups(zip(models.words, first, rows_of))
        self.tenant = ints(np.repeat(np.arange(len(self.rows_of)), rows_of), dev)
        self.token = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.x, self.normed, self.qkv, self.seen, self.added = buf(w), buf(w), buf(q + 2 * kv), buf(q), buf(w)
        self.logits = buf(models.vocabulary, torch.float32)
        self.uniform, self.samples = torch.zeros(rows, device=dev), mt.alloc_samples(rows, models.vocabulary, device=dev)


class Models:
    """The tenants' models and their cache.  weights[t]: {"embedding" [vocabulary, width], "words" [vocabulary, width], "layers": [{"qkv", "out", "gain"}], "gain"}, fp32."""

    def __init__(self, weights, heads, kv_heads, head_dim, seqs, tokens, page=16, kv8=True, device="cuda:0"):
        self.device, self.heads, self.kv_heads, self.head_dim = device, heads, kv_heads, head_dim
        self.q_width, self.kv_width, self.width = heads * head_dim, kv_heads * head_dim, weights[0]["embedding"].shape[1]
        self.vocabulary = weights[0]["embedding"].shape[0]
        need = sum(mt.matrix4_footprint(*m.shape) for one in weights for m in [one["words"], *(layer[n] for layer in one["layers"] for n in ("qkv", "out"))])
        self.ctx = mt.Context(1, 1, 64, 1, need + (1 << 20), mt.MT_BF16, torch.device(device).index or 0)
        put = lambda m: self.ctx.register_matrix4(*m.shape, *to_4_bits(m))  # noqa: E731
        gains = lambda pick: torch.from_numpy(np.stack([pick(one) for one in weights])).to(device)  # noqa: E731
        self.layers = [{"qkv": [put(one["layers"][i]["qkv"]) for one in weights], "out": [put(one["layers"][i]["out"]) for one in weights], "gain": gains(lambda one: one["layers"][i]["gain"])}
                       for i in range(len(weights[0]["layers"]))]
        self.words, self.gain = [put(one["words"]) for one in weights], gains(lambda one: one["gain"])
        self.embedding = gains(lambda one: one["embedding"]).to(torch.bfloat16)
        width = -(-tokens // page)
        self.cache = mt.alloc_kv(seqs * (width + 1), page, kv_heads, head_dim, seqs, width, dtype=mt.MT_KV8 if kv8 else mt.MT_BF16, layers=len(self.layers), device=device)
        self.reach = width * page

    def run(self, r, seqs, first_row=None, max_new=1, scratch=None, **settings):
        """The layers for r's rows (the last tokens of `seqs`, which their lengths count already), and a token drawn behind each."""
        ctx, c, q, kv = self.ctx, self.cache, self.q_width, self.kv_width
        r.x.copy_(self.embedding[r.tenant.long(), r.token.long()])
        for i, layer in enumerate(self.layers):
            # (the stream of the layer before is added on the way)
            mt.add_norm(ctx, r.x, residual=r.added if i else None, gain=layer["gain"], gain_ids=r.tenant, sum_out=r.x if i else None, out=r.normed)
            mt.linear4(ctx, r.groups[i][0], r.normed, r.qkv)
            mt.kv_write(ctx, c, r.qkv[:, q:q + kv], r.qkv[:, q + kv:], seqs=seqs, first_row=first_row, max_new=max_new, layer=i)
            mt.attend(ctx, c, r.qkv[:, :q], r.seen, seqs=seqs, first_row=first_row, max_new=max_new, max_length=self.reach, layer=i, scratch=scratch)
            mt.linear4(ctx, r.groups[i][1], r.seen, r.added)
        mt.add_norm(ctx, r.x, residual=r.added, gain=self.gain, gain_ids=r.tenant, out=r.normed)
        mt.linear4(ctx, r.word_groups, r.normed, r.logits)
        return mt.sample(ctx, r.logits, r.uniform, r.samples, **settings)

    def scratch(self, n_seqs, max_new=1):
        return mt.alloc_attend(self.ctx, self.cache, self.heads, n_seqs, max_new, self.reach)

    def close(self):
        self.ctx.close()


class Answers:
    """`answers` answers to every prompt (a list of tokens), prompts[t] those of tenant t; settings: lists of a value for every answer."""

    def __init__(self, models, prompts, answers, settings, seed=0):
        m, dev = models, models.device
        self.models, self.rng = m, np.random.default_rng(seed)
        flat = [p for t in prompts for p in t]
        n = len(flat)
        # the prompts go in whole: sequences 0 .. n - 1
        lengths = [len(p) for p in flat]
        first = np.concatenate([[0], np.cumsum(lengths)])
        r = Rows(m, [sum(len(p) for p in t) for t in prompts])
        r.token.copy_(ints([v for p in flat for v in p], dev))
        self.granted = ints([0] * n, dev)
        mt.kv_grow(m.ctx, m.cache, ints(lengths, dev), granted=self.granted)
        seqs = ints(range(n), dev)
        r.uniform.copy_(torch.from_numpy(self.rng.random(int(first[-1])).astype(np.float32)))
        m.run(r, seqs, ints(first, dev), max(lengths), m.scratch(n, max(lengths)))
        self.prompt_rows = r
        # every answer but a prompt's first is a fork
        owner = np.repeat(np.arange(n), answers)
        self.seqs = ints([p if i % answers == 0 else n + i - p - 1 for i, p in enumerate(owner)], dev)
        forks = [i for i in range(n * answers) if i % answers]
        if forks:
            mt.kv_fork(m.ctx, m.cache, ints(owner[forks], dev), self.seqs[torch.tensor(forks, device=dev)])
        self.rows = Rows(m, [len(t) * answers for t in prompts])
        self.settings = {k: (torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32)).to(dev) for k, v in settings.items()}
        # their first tokens: drawn from what the prompts' last rows said
        last = torch.from_numpy(first[1:][owner] - 1).to(dev)
        self.rows.uniform.copy_(torch.from_numpy(self.rng.random(n * answers).astype(np.float32)))
        mt.sample(m.ctx, r.logits[last].contiguous(), self.rows.uniform, self.rows.samples, **self.settings)
        self.one, self.scratch, self.graph = ints([1] * (n * answers), dev), m.scratch(n * answers), None
        self.tokens = [self.rows.samples.ids.clone()]

    def launch(self):
        self.rows.token.copy_(self.rows.samples.ids)
        mt.kv_grow(self.models.ctx, self.models.cache, self.one, seqs=self.seqs)
        self.models.run(self.rows, self.seqs, scratch=self.scratch, **self.settings)

    def step(self):
        """One more token of every answer."""
        self.rows.uniform.copy_(torch.from_numpy(self.rng.random(len(self.one)).astype(np.float32)))
        if self.graph is None:
            self.launch()
            torch.cuda.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.launch()
        else:
            self.graph.replay()
        self.tokens.append(self.rows.samples.ids.clone())

    def drop(self):
        """The answers leave; what others hold moves together."""
        self.graph = None
        mt.kv_free(self.models.ctx, self.models.cache, self.seqs)
        mt.kv_compact(self.models.ctx, self.models.cache)


def random_models(rng, tenants, layers, heads, kv_heads, head_dim, vocabulary):
    width = heads * head_dim
    draw = lambda *shape: rng.standard_normal(shape, dtype=np.float32) * shape[-1] ** -0.5  # noqa: E731
    gain = lambda: 1 + 0.1 * rng.standard_normal(width, dtype=np.float32)  # noqa: E731
    return [{"embedding": draw(vocabulary, width) * width ** 0.5, "words": 4 * draw(vocabulary, width), "gain": gain(),
             "layers": [{"qkv": 2 * draw((heads + 2 * kv_heads) * head_dim, width), "out": draw(width, width), "gain": gain()} for _ in range(layers)]} for _ in range(tenants)]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("tenants", 4), ("answers", 2), ("prompt", 200), ("tokens", 32), ("layers", 2), ("heads", 8), ("kv_heads", 2), ("head_dim", 64), ("vocabulary", 8192)):
        p.add_argument("--" + name, type=int, default=default)
    a = p.parse_args(argv)
    rng = np.random.default_rng(0)
    models = Models(random_models(rng, a.tenants, a.layers, a.heads, a.kv_heads, a.head_dim, a.vocabulary), a.heads, a.kv_heads, a.head_dim, a.tenants * a.answers, a.prompt + a.tokens)
    prompts = [[rng.integers(0, a.vocabulary, max(1, a.prompt - 7 * t)).tolist()] for t in range(a.tenants)]
    n = a.tenants * a.answers
    run = Answers(models, prompts, a.answers, {"temperature": [0.0 if i % a.answers == 0 else 0.8 for i in range(n)], "top_k": [50] * n, "top_p": [0.95] * n})
    run.step(), run.step()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.tokens - 3):
        run.step()
    torch.cuda.synchronize()
    print("%d answers of %d tenants: %.1f us a token" % (n, a.tenants, (time.perf_counter() - start) / max(a.tokens - 3, 1) * 1e6), flush=True)
    tokens = torch.stack(run.tokens, 1).tolist()
    for i in range(n):
        print("tenant %d: %s" % (i // a.answers, tokens[i][:12]))
    run.drop()
    print("pages held behind all of them: %d" % int((models.cache.refs > 0).sum()))
    models.close()


if __name__ == "__main__":
    main()
