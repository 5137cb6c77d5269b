"""The example that runs the calls on caches together, launch by launch against 64 bits, and the whole against a cache-less evaluation."""
import os
import sys

import numpy as np
import pytest
import torch

import lm_cache_common as lc
import lm_common as lm

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def cached(c, layer, s, length):
    """Keys and values [tokens, heads, dim] of a sequence, in 64 bits, by its table."""
    page = c.k.shape[3]
    t = np.arange(length)
    p, slot = c.table[s].long().cpu().numpy()[t // page], t % page
    out = []
    for x, scales, turned in ((c.k, c.k_scales, False), (c.v, c.v_scales, True)):
        v = lm.e4m3(x[layer].view(torch.uint8).cpu().numpy()) if scales is not None else lc.in_64(x[layer])
        v = v[p, :, :, slot] if turned else v[p, :, slot]
        if scales is not None:
            v = v * lm.e8m0(scales[layer].view(torch.uint8).cpu().numpy()[p, :, slot])[..., None]
        out.append(v)
    return out


@pytest.mark.parametrize("kv8", [False, True])
def test_answers_of_several_tenants(kv8):
    import decode
    rng = np.random.default_rng(4)
    heads, kv_heads, dim, vocabulary, answers, layers = 4, 2, 64, 777, 3, 2
    prompts = [[rng.integers(0, vocabulary, n).tolist() for n in t] for t in ([33, 5], [16], [1, 70])]
    n = 5 * answers
    models = decode.Models(decode.random_models(rng, 3, layers, heads, kv_heads, dim, vocabulary), heads, kv_heads, dim, n, 100, kv8=kv8)
    settings = {"temperature": [0.0, 1.0, 0.7] * 5, "top_k": [0, 40, 0] * 5, "top_p": [1.0, 0.9, 0.95] * 5, "min_p": [0.0, 0.0, 0.02] * 5}
    run = decode.Answers(models, prompts, answers, settings, seed=1)
    c, q, kv, scale = models.cache, models.q_width, models.kv_width, float(np.float32(dim ** -0.5))
    assert run.granted.tolist() == [1] * 5
    seqs, lengths = run.seqs.tolist(), [len(p) for t in prompts for p in t for _ in range(answers)]
    assert sorted(seqs) == list(range(n)) and [c.lengths[s].item() for s in seqs] == lengths
    # full pages are shared, last ones are not
    table, refs = c.table.cpu().numpy(), c.refs.cpu().numpy()
    for first in range(0, n, answers):
        for i, s in enumerate(seqs[first:first + answers]):
            for j in range(-(-lengths[first] // 16)):
                whole = (j + 1) * 16 <= lengths[first]
                assert (table[s, j] == table[seqs[first], j]) == (whole or i == 0) and refs[table[s, j]] == (answers if whole else 1)
    forked = {(layer, s): cached(c, layer, s, lengths[i]) for layer in range(layers) for i, s in enumerate(seqs)}
    for i in range(n):
        for layer in range(layers):
            for a, b in zip(forked[layer, seqs[i]], forked[layer, seqs[i // answers * answers]]):
                assert np.array_equal(a, b)
    for step in range(5):
        run.step()
        torch.cuda.synchronize()
        lengths = [v + 1 for v in lengths]
        r = run.rows
        assert [c.lengths[s].item() for s in seqs] == lengths and torch.equal(r.token, run.tokens[-2])
        # the last layer: what it wrote, what it saw
        new = lc.in_64(r.qkv)
        for i, s in enumerate(seqs):
            k, v = cached(c, layers - 1, s, lengths[i])
            for got, put in ((k, new[i, q:q + kv]), (v, new[i, q + kv:])):
                put = put.reshape(kv_heads, dim)
                assert np.array_equal(got[-1], lc.values_of(lc.in_8_bits(put)) if kv8 else put)
            for got, before in zip((k, v), forked[layers - 1, s]):
                assert np.array_equal(got[:len(before)], before)
            out, _, off, _ = lc.attended(new[i, :q].reshape(heads, dim), k, v, 0, lengths[i], scale, "bf16")
            assert np.all(np.abs(lc.in_64(r.seen[i]).reshape(heads, dim) - out) <= off)
        # what it said, and what was drawn
        logits, ids, u = lc.in_64(r.logits), r.samples.ids.tolist(), r.uniform.cpu().numpy()
        for i in range(n):
            want = lc.sampled(logits[i], u[i], **{k: (w[i] if k == "top_k" else np.float32(w[i])) for k, w in settings.items()})
            assert ids[i] == want[0] and int(r.samples.kept[i]) == want[2]
    run.drop()
    torch.cuda.synchronize()
    assert not c.refs.any() and not c.lengths.any()
    # greedy answers are what the same tokens give as a prompt, without a cache from before
    tokens = torch.stack(run.tokens, 1).tolist()
    again = decode.Answers(models, [[p + tokens[answers * j][:-1]] for j, p in zip((0, 2, 3), (prompts[0][0], prompts[1][0], prompts[2][0]))], 1, {"temperature": [0.0] * 3}, seed=2)
    last = lc.in_64(again.prompt_rows.logits[torch.cumsum(torch.tensor(again.prompt_rows.rows_of), 0).cuda() - 1])
    for i, j in enumerate((0, 2, 3)):
        # (bf16 streams, and in 8 bits other pages' scales: the same token, unless the best two are as near as such roundings)
        top = np.sort(last[i])[-2:]
        assert tokens[answers * j][-1] == int(last[i].argmax()) or top[1] - top[0] < 0.1
    models.close()
