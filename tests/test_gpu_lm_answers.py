"""The example that runs the operators together, launch by launch against 64 bits."""
import os
import sys

import numpy as np
import pytest
import torch

import lm_common as lm

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def values(q, scales):
    return lm.e4m3(q.view(torch.uint8).cpu().numpy()) * lm.spread(lm.e8m0(scales.view(torch.uint8).cpu().numpy()), q.shape[1])


def in_64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows_of,width,hidden,vocabulary", [([1], 64, 96, 500), ([3, 0, 17, 1], 321, 200, 10001), ([2, 33, 5], 1024, 1024, 4096)])
def test_the_step_of_several_tenants(rows_of, width, hidden, vocabulary):
    import answers
    rng = np.random.default_rng(width)
    layers, gains = answers.random_tenants(rng, len(rows_of), width, hidden, vocabulary)
    step = answers.AnswerStep(layers, gains, rows_of, top=4, temperature=0.8)
    rows, tenant = sum(rows_of), np.repeat(np.arange(len(rows_of)), rows_of)
    weights = []
    for one in layers:
        weights.append([])
        for w in (one[0], one[2], one[3]):
            codes, scales = answers.to_4_bits(w)
            c = np.stack((codes & 15, codes >> 4), -1).reshape(w.shape[0], -1)[:, :w.shape[1]]
            weights[-1].append(lm.E2M1[c] * lm.spread(lm.e8m0(scales), w.shape[1]))
            assert np.all(np.abs(weights[-1][-1] - w) <= lm.spread(lm.e8m0(scales), w.shape[1]))          # half of the widest step, 2
    n_words = np.array([w[2].shape[0] for w in weights])[tenant]
    for again in range(3):
        step.x.copy_(torch.from_numpy(rng.standard_normal((rows, width))))
        step.delta.copy_(torch.from_numpy(rng.standard_normal((rows, width))))
        step.next.copy_(torch.from_numpy(rng.integers(0, n_words, rows).astype(np.int32).reshape(rows, 1)))
        o = step.run()
        torch.cuda.synchronize()
        # every launch from what the one before left: bf16 rounds by 2^-9 of a value, e4m3 by 2^-4 or half its smallest step
        h = in_64(step.x) + in_64(step.delta)
        assert np.all(np.abs(in_64(step.h) - h) <= 2.0 ** -8 * np.abs(h))
        for q, scales, sums in ((step.q, step.q_scales, h), (step.q2, step.q2_scales, in_64(step.h) + in_64(step.d))):
            y = sums / np.sqrt((sums * sums).mean(1, keepdims=True) + 1e-6) * np.stack(gains)[tenant]
            s = lm.spread(lm.e8m0(scales.view(torch.uint8).cpu().numpy()), width)
            assert np.all(np.abs(values(q, scales) - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s) * (1 + 1e-5) + 1e-5 * np.abs(y))
        for pick, x, got, dtype in ((0, values(step.q, step.q_scales), step.mid, "bf16"), (1, in_64(step.mid), step.d, "bf16"), (2, values(step.q2, step.q2_scales), step.logits, "f32")):
            for r in range(rows):
                w = weights[tenant[r]][pick]
                z, size = w @ x[r], np.abs(w) @ np.abs(x[r])
                if pick == 0:
                    z = z + layers[tenant[r]][1]
                    size = size + np.abs(layers[tenant[r]][1])
                want = in_64(torch.nn.functional.gelu(torch.from_numpy(z))) if pick == 0 else z
                # sums of at most 1024 products in fp32, each addition off by 2^-24 of what it has; GELU's slope is below 1.13
                near = 1024 * 2.0 ** -24 * size * 1.13 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0) + 1e-6
                assert np.all(np.abs(in_64(got[r, :len(want)]) - want) <= near), (again, pick, r)
        ref = lm.scored(in_64(step.logits), n_words, None, step.next.cpu().numpy(), 4, float(np.float32(0.8)))
        assert np.array_equal(o.top_ids.cpu().numpy(), ref["ids"]) and np.array_equal(o.given_ranks.cpu().numpy(), ref["ranks"])
        for got, want in ((o.entropy, ref["entropy"]), (o.given_logprobs, ref["given"]), (o.top_logprobs, ref["top"])):
            bound = ref["bound"] if want.ndim == 1 else ref["bound"][:, None]
            assert np.all(np.abs(in_64(got) - want) <= bound + 2.0 ** -21 * np.abs(want))
    step.close()


@pytest.mark.parametrize("what", ["norm", "layer", "scores"])
def test_written_tensors_count_as_changed(what):
    """What a graph of gradients has saved may not be overwritten without a word."""
    import paper_1901_06887_amd as mt
    ctx = mt.Context(1, 1, 64, 1, 1 << 20, mt.MT_BF16, 0)
    x, w = torch.randn(4, 32, device="cuda"), torch.ones(4, 32, device="cuda", requires_grad=True)
    out = torch.ones(4, 32, device="cuda")
    loss = (w * out).sum()
    if what == "norm":
        mt.add_norm(ctx, x, out=out)
    elif what == "layer":
        m = ctx.register_matrix4(32, 32, np.full((32, 16), 0x22, dtype=np.uint8), np.full((32, 1), 127, dtype=np.uint8))
        mt.linear4(ctx, mt.row_groups([(m, 0, 4)]), x, out)
    else:
        o = mt.alloc_scores(4, 0, 32)
        o.top_logprobs = out
        mt.score(ctx, x, o)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():            # (tensors that carry no versions)
        a = torch.ones(4, 32, device="cuda")
    mt.add_norm(ctx, x, out=a)
    ctx.close()
