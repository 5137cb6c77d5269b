"""What the operators behind language models' answers are measured on: the norm in front of a 4-bit layer, the layer, and the scores of its classes.

A pass is one call of one operator.  Where `own` is false it is computed in its plain form, elementary torch operations in 32 bits; where it
is true, by the runtime's entry point, on the same inputs and into buffers that the caller holds.

The keys of a case
  op        norm: h = x + residual; y = h / sqrt(mean(h^2) + eps) * gain, as it is and in 8 bits with scales
            linear: y = act(x W^T + bias) for the rows of each of several tenants, W in 4 bits with scales
            score: of every row's classes: log probabilities and ranks of given ones, entropy, the best alternatives
  norm      rows, width, dtype (bf16, f32), residual, gains (tenants with a gain of their own; a row names its tenant),
            y (write y in dtype), q (write y in 8 bits: e4m3 with a power of two for every 32 values)
  linear    tenants; lo, hi (rows of each: spread over lo..hi); k, n (in and out features); x (bf16, f32, or mx8: e4m3 with a power of
            two for every 32 values), y (bf16, f32), act (none, relu, gelu), bias.  Weights: e2m1 with a power of two for every 32 values
  score     rows, classes, dtype (bf16, f32), given, top, masked (a bit for each class says whether it is allowed), ragged (rows have
            class counts of their own), temperature
"""
import math

import torch

own = False
EPS = 1e-6
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    norm, linear, score = {"op": "norm"}, {"op": "linear"}, {"op": "score"}
    return [
        # one token of one tenant between two layers of a small model: latency
        dict(norm, name="norm_one_row", rows=1, width=1024, dtype="bf16", residual=True, gains=1, y=False, q=True),
        # rows of many tenants, each with its gain, at a width that fits no vector
        dict(norm, name="norm_f32_odd", rows=333, width=1531, dtype="f32", residual=True, gains=24, y=True, q=True),
        # a long prompt, or the prompts of many tenants: memory decides
        dict(norm, name="norm_prompt", rows=8192, width=4096, dtype="bf16", residual=True, gains=8, y=True, q=True),
        # one token through a small hidden layer: latency
        dict(linear, name="linear_one_row", tenants=1, lo=1, hi=1, k=1024, n=1024, x="bf16", y="bf16", act="gelu", bias=True),
        # one token through the last layer of a large vocabulary: the weights' bytes
        dict(linear, name="linear_vocab_one_row", tenants=1, lo=1, hi=1, k=4096, n=65536, x="bf16", y="f32", act="none", bias=False),
        # a step of many tenants with a few tokens each
        dict(linear, name="linear_many_tenants", tenants=64, lo=1, hi=4, k=1024, n=1024, x="mx8", y="bf16", act="relu", bias=True),
        # a step of a few tenants with full batches through wide hidden layers
        dict(linear, name="linear_batches", tenants=8, lo=37, hi=64, k=4096, n=4096, x="mx8", y="bf16", act="gelu", bias=True),
        # one tenant's prompt: arithmetic counts too
        dict(linear, name="linear_prompt", tenants=1, lo=512, hi=512, k=4096, n=4096, x="bf16", y="bf16", act="none", bias=True),
        # fp32 rows through sizes that fit no tile
        dict(linear, name="linear_f32_odd", tenants=5, lo=3, hi=11, k=301, n=333, x="f32", y="f32", act="relu", bias=True),
        # the answer to one request, of the classes of the residual nets: latency
        dict(score, name="score_one_row", rows=1, classes=1000, dtype="f32", given=1, top=5, masked=False, ragged=False, temperature=1.0),
        # a step of sixteen requests whose answers a grammar restricts, several candidates each
        dict(score, name="score_masked_step", rows=16, classes=65001, dtype="bf16", given=4, top=20, masked=True, ragged=True, temperature=0.7),
        # every token of a prompt scored: memory decides
        dict(score, name="score_prompt", rows=2048, classes=32768, dtype="f32", given=1, top=1, masked=False, ragged=False, temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, multiple):
    """A size spread over its logarithm; half of them round, half as they come."""
    v = _log_int(rng, lo, hi)
    return max(multiple, v // multiple * multiple) if rng.random() < 0.5 else v


def draw(rng):
    while True:
        op = rng.choice(("norm", "linear", "linear", "score"))
        if op == "norm":
            c = {"op": op, "rows": _log_int(rng, 1, 8192), "width": _size(rng, 64, 8192, 64), "dtype": rng.choice(("bf16", "f32")),
                 "residual": rng.random() < 0.7, "gains": rng.choice((1, 1, 8, 24, 64)), "y": rng.random() < 0.6}
            c["q"] = not c["y"] or rng.random() < 0.6
            fits = c["rows"] * c["width"] * (1 if c["dtype"] == "bf16" else 2) <= 8192 * 4096
        elif op == "linear":
            c = {"op": op, "tenants": _log_int(rng, 1, 64), "lo": _log_int(rng, 1, 64), "k": _size(rng, 64, 8192, 64), "n": _size(rng, 10, 65536, 64),
                 "x": rng.choice(("bf16", "bf16", "mx8", "mx8", "f32")), "y": rng.choice(("bf16", "f32")), "act": rng.choice(("none", "relu", "gelu")),
                 "bias": rng.random() < 0.6}
            c["hi"] = _log_int(rng, c["lo"], 512 if c["tenants"] == 1 else max(c["lo"], 64))
            macs = c["k"] * c["n"] * c["tenants"]
            fits = macs <= 4096 * 65536 and macs * c["hi"] <= 4096 * 4096 * 512
        else:
            c = {"op": op, "rows": _log_int(rng, 1, 2048), "classes": _size(rng, 10, 131072, 64), "dtype": rng.choice(("bf16", "f32")),
                 "given": rng.choice((0, 1, 1, 2, 4, 8)), "top": rng.choice((0, 1, 5, 8, 20)), "masked": rng.random() < 0.3, "ragged": rng.random() < 0.4,
                 "temperature": rng.choice((1.0, 1.0, 0.7, 1.3))}
            fits = c["rows"] * c["classes"] <= 2048 * 32768
        if fits:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _rows_of(case):
    """Rows of every tenant, spread over lo..hi."""
    span = case["hi"] - case["lo"] + 1
    return [case["lo"] + (t * 7919 + 5) % span if span > 1 else case["lo"] for t in range(case["tenants"])]


def _e8m0(exponent):
    return (exponent + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _blocks(x):
    """[..., k] with zeros up to a multiple of 32, as [..., blocks, 32]."""
    pad = -x.shape[-1] % 32
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, 32))


def _exponent(amax, largest, octave):
    """The least e with amax <= largest * 2^octave * 2^e, largest in [0.5, 1); 0 where amax is 0."""
    m, e = torch.frexp(amax)
    e = e - octave + (m > largest).to(e.dtype)
    return torch.where(amax > 0, e.clamp(-126, 127), torch.zeros_like(e))


def _power(e):
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _in_8_bits(y):
    """e4m3 values and e8m0 scales of rows of fp32: the least power of two for every 32 values at which none exceeds 448."""
    b = _blocks(y)
    e = _exponent(b.abs().amax(-1), 0.875, 9)
    q = (b * _power(-e).unsqueeze(-1)).flatten(-2)[..., :y.shape[-1]]
    return q.to(torch.float8_e4m3fn), _e8m0(e)


def _in_4_bits(w):
    """Packed e2m1 codes (the even column in the low half) and e8m0 scales of fp32 weights [..., n, k]."""
    k = w.shape[-1]
    b = _blocks(w)
    e = _exponent(b.abs().amax(-1), 0.75, 3)
    s = (b * _power(-e).unsqueeze(-1)).flatten(-2)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    codes = torch.bucketize(s.abs(), edges, out_int32=True).to(torch.uint8) | ((s < 0).to(torch.uint8) << 3)
    codes = codes[..., :k + k % 2]
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).contiguous(), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 1000003 + 17)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    uniform = lambda hi, *shape: torch.randint(hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    s = {"case": case}
    if case["op"] == "norm":
        R, D, dt = case["rows"], case["width"], DTYPES[case["dtype"]]
        wide = torch.where(torch.rand(D, generator=g, device="cuda") < 0.01, 20.0, 1.0)            # a few channels stand out, as in residual streams
        s["x"] = (randn(R, D) * wide).to(dt)
        s["residual"] = (randn(R, D) * 0.3 * wide).to(dt) if case["residual"] else None
        s["gain"] = 1.0 + 0.2 * randn(case["gains"], D)
        s["ids"] = uniform(case["gains"], R) if case["gains"] > 1 else None
        if own:
            s["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
            s["y"] = torch.empty_like(s["x"]) if case["y"] else None
            s["q"] = torch.empty(R, D, dtype=torch.float8_e4m3fn, device="cuda") if case["q"] else None
            s["scales"] = torch.empty(R, -(-D // 32), dtype=torch.float8_e8m0fnu, device="cuda") if case["q"] else None
    elif case["op"] == "linear":
        T, K, N, counts = case["tenants"], case["k"], case["n"], _rows_of(case)
        R = sum(counts)
        codes, scales, bias = [], [], []
        for _ in range(T):
            c, e = _in_4_bits(randn(N, K) * K ** -0.5)
            codes.append(c), scales.append(e), bias.append(0.1 * randn(N))
        codes, scales, bias = torch.stack(codes), torch.stack(scales), torch.stack(bias)
        x = randn(R, K)
        s["x"], s["x_scales"] = _in_8_bits(x) if case["x"] == "mx8" else (x.to(DTYPES[case["x"]]), None)
        first = [sum(counts[:t]) for t in range(T)]
        if own:
            s["matrices"] = _register(s, codes, scales, bias if case["bias"] else None, K)
            s["groups"] = _groups(s["matrices"], first, counts)
            s["out"] = torch.empty(R, N, dtype=DTYPES[case["y"]], device="cuda")
        else:
            s["codes"], s["scales"], s["bias"] = codes, scales, bias if case["bias"] else None
            s["tenant"] = torch.repeat_interleave(torch.arange(T), torch.tensor(counts)).cuda()    # of every row, and its place among the tenant's
            s["place"] = torch.cat([torch.arange(n) for n in counts]).cuda()
    else:
        R, C = case["rows"], case["classes"]
        s["logits"] = (2.5 * randn(R, C) + 9.0 * (torch.rand(R, C, generator=g, device="cuda") < 4.0 / C)).to(DTYPES[case["dtype"]])
        s["n"] = (C - uniform(C // 4 + 1, R)).to(torch.int32) if case["ragged"] else None
        s["allowed"] = uniform(1 << 16, R, -(-C // 32)) | (uniform(1 << 15, R, -(-C // 32)) << 16) if case["masked"] else None
        s["given"] = (torch.rand(R, case["given"], generator=g, device="cuda") * (s["n"].unsqueeze(1) if case["ragged"] else C)).to(torch.int32) if case["given"] else None
        if own:
            import paper_1901_06887_amd as mt
            s["out"] = mt.alloc_scores(R, case["given"], case["top"], device=s["logits"].device)
    if own and "ctx" not in s:
        s["ctx"] = _context(1 << 16)
    return s


def _context(arena_bytes):
    import paper_1901_06887_amd as mt
    return mt.Context(1, 1, 64, 1, arena_bytes, mt.MT_BF16, torch.cuda.current_device())


def _register(s, codes, scales, bias, k):
    """The tenants' matrices in a context's arena; their numbers."""
    import paper_1901_06887_amd as mt
    T, N = codes.shape[0], codes.shape[1]
    s["ctx"] = _context(T * mt.matrix4_footprint(N, k) + (1 << 20))
    codes, scales, bias = codes.cpu().numpy(), scales.cpu().numpy(), bias.cpu().numpy() if bias is not None else [None] * T
    return [s["ctx"].register_matrix4(N, k, codes[t], scales[t], bias[t]) for t in range(T)]


def _groups(matrices, first, counts):
    import paper_1901_06887_amd as mt
    return mt.row_groups(zip(matrices, first, counts))


# ---- the operators ----------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state, state["case"])


def _own_norm(s, case):
    import paper_1901_06887_amd as mt
    mt.add_norm(s["ctx"], s["x"], s["residual"], s["gain"], s["ids"], eps=EPS, sum_out=s["sum"], out=s["y"], out8=s["q"], out8_scales=s["scales"])
    return {"sum": s["sum"], "y": s["y"], "q": s["q"], "scales": s["scales"]}


def _own_linear(s, case):
    import paper_1901_06887_amd as mt
    act = {"none": mt.MT_ACT_NONE, "relu": mt.MT_ACT_RELU, "gelu": mt.MT_ACT_GELU}[case["act"]]
    mt.linear4(s["ctx"], s["groups"], s["x"], s["out"], x_scales=s["x_scales"], act=act)
    return s["out"]


def _own_score(s, case):
    import paper_1901_06887_amd as mt
    o = mt.score(s["ctx"], s["logits"], s["out"], given=s["given"], n_classes=s["n"], allowed=s["allowed"], temperature=case["temperature"])
    return {"entropy": o.entropy, "given": o.given_logprobs, "ranks": o.given_ranks, "ids": o.top_ids, "top": o.top_logprobs}


def _plain_norm(s, case):
    h = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    gain = s["gain"] if s["ids"] is None else s["gain"][s["ids"]]
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * gain
    q, scales = _in_8_bits(y) if case["q"] else (None, None)
    dt = DTYPES[case["dtype"]]
    return {"sum": h.to(dt) if case["residual"] else None, "y": y.to(dt) if case["y"] else None, "q": q, "scales": scales}


def _plain_linear(s, case):
    K, dev = case["k"], s["x"].device
    codes = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).flatten(-2)[..., :K]
    w = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=dev)[codes.to(torch.int32)]
    w = w * _power(s["scales"].to(torch.int32) - 127).repeat_interleave(32, -1)[..., :K]
    x = s["x"].float()
    if s["x_scales"] is not None:
        x = x * _power(s["x_scales"].view(torch.uint8).to(torch.int32) - 127).repeat_interleave(32, -1)[..., :K]
    columns = torch.zeros(case["tenants"], K, case["hi"], device=dev)
    columns[s["tenant"], :, s["place"]] = x
    y = torch.bmm(w, columns)[s["tenant"], :, s["place"]]
    if s["bias"] is not None:
        y = y + s["bias"][s["tenant"]]
    if case["act"] == "relu":
        y = torch.clamp(y, min=0)
    elif case["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * 0.5 ** 0.5))
    return y.to(DTYPES[case["y"]])


def _allowed(s, classes):
    """Which classes of every row count."""
    j = torch.arange(classes, device=s["logits"].device)
    ok = torch.ones(s["logits"].shape, dtype=torch.bool, device=j.device) if s["n"] is None else j < s["n"].unsqueeze(1)
    return ok if s["allowed"] is None else ok & ((s["allowed"][:, j // 32] >> (j % 32).to(torch.int32)) & 1).bool()


def _plain_score(s, case):
    C, none = case["classes"], -math.inf
    x = s["logits"].float()
    x = torch.where(_allowed(s, C), x, none)
    z = (x - x.amax(1, keepdim=True)) * (1.0 / case["temperature"])
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    o = {"entropy": (log_total - torch.where(e > 0, z * e, 0.0).sum(1, keepdim=True) / total).squeeze(1), "given": None, "ranks": None, "ids": None, "top": None}
    if s["given"] is not None:
        j, given = torch.arange(C, device=x.device), s["given"].long()
        o["given"] = z.gather(1, given) - log_total
        at = x.gather(1, given)
        ranks = [((x > at[:, i:i + 1]) | ((x == at[:, i:i + 1]) & (j < given[:, i:i + 1]))).sum(1) for i in range(case["given"])]
        o["ranks"] = torch.where(at > none, torch.stack(ranks, 1), -1).to(torch.int32)
    if case["top"]:
        v, ids = (t[:, :case["top"]] for t in torch.sort(x, dim=1, descending=True, stable=True))
        o["ids"] = torch.nn.functional.pad(torch.where(v > none, ids, -1), (0, case["top"] - v.shape[1]), value=-1).to(torch.int32)
        o["top"] = torch.nn.functional.pad(z.gather(1, ids) - log_total, (0, case["top"] - v.shape[1]), value=none)
    return o


_own = {"norm": _own_norm, "linear": _own_linear, "score": _own_score}
_plain = {"norm": _plain_norm, "linear": _plain_linear, "score": _plain_score}


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits; 8-bit values before their rounding.  Whole numbers are held to be equal and left out here."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "norm":
        h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        root = (h.pow(2).sum(-1, keepdim=True) / case["width"] + EPS).sqrt()
        y = h / root * (s["gain"].double() if s["ids"] is None else s["gain"].double()[s["ids"]])
        q = scales = None
        if case["q"]:
            most = torch.nn.functional.pad(y, (0, -case["width"] % 32)).abs().view(case["rows"], -1, 32).max(-1).values
            scales = torch.where(most > 0, torch.exp2(torch.ceil(torch.log2(most / 448.0))), 1.0)
            q = y / torch.repeat_interleave(scales, 32, dim=1)[:, :case["width"]]
        return {"sum": h if case["residual"] else None, "y": y if case["y"] else None, "q": q, "scales": scales}
    if case["op"] == "linear":
        at, rows = 0, []
        value = torch.tensor([(-1.0 if c & 8 else 1.0) * (0.5 * (c & 1) if not c & 6 else (1 + 0.5 * (c & 1)) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)],
                             dtype=torch.float64, device=s["x"].device)
        scale = lambda bits: torch.exp2(bits.view(torch.uint8).double() - 127)  # noqa: E731
        x = s["x"].double()
        if s["x_scales"] is not None:
            x = x * scale(s["x_scales"]).repeat_interleave(32, 1)[:, :case["k"]]
        for t, n in enumerate(_rows_of(case)):
            c = s["codes"][t].int()
            w = torch.empty(case["n"], 2 * c.shape[1], dtype=torch.float64, device=x.device)
            w[:, 0::2], w[:, 1::2] = value[c & 15], value[c >> 4]
            w = w[:, :case["k"]] * scale(s["scales"][t]).repeat_interleave(32, 1)[:, :case["k"]]
            y = x[at:at + n] @ w.t()
            at += n
            y = y + s["bias"][t].double() if case["bias"] else y
            rows.append(y.clamp(min=0) if case["act"] == "relu" else y * torch.special.ndtr(y) if case["act"] == "gelu" else y)
        return torch.cat(rows)
    o = {"entropy": [], "given": [], "ranks": None, "ids": None, "top": []}
    for r in range(case["rows"]):
        x = s["logits"][r].double() / case["temperature"]
        n = case["classes"] if s["n"] is None else int(s["n"][r])
        if case["masked"]:
            bits = s["allowed"][r].view(torch.uint8).unsqueeze(1) >> torch.arange(8, device=x.device, dtype=torch.uint8) & 1
            x = torch.where(bits.flatten()[:case["classes"]].bool(), x, -math.inf)
        x = torch.where(torch.arange(case["classes"], device=x.device) < n, x, -math.inf)
        lp = torch.log_softmax(x, 0)
        o["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum())
        if case["given"]:
            o["given"].append(lp[s["given"][r].long()])
        if case["top"]:
            v = torch.topk(lp, min(case["top"], case["classes"])).values
            o["top"].append(torch.nn.functional.pad(v, (0, case["top"] - v.shape[0]), value=-math.inf))
    return {k: torch.stack(v) if v else None for k, v in o.items()}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        R, D, es = case["rows"], case["width"], 2 if case["dtype"] == "bf16" else 4
        touched = es * (1 + 2 * case["residual"] + case["y"]) + case["q"] * (1 + 1 / 32)
        return {"bytes": R * D * touched + 4 * D * min(case["gains"], R) + (4 * R if case["gains"] > 1 else 0), "flops": 6 * R * D}
    if case["op"] == "linear":
        T, K, N, R = case["tenants"], case["k"], case["n"], sum(_rows_of(case))
        x = {"bf16": 2, "f32": 4, "mx8": 1 + 1 / 32}[case["x"]]
        weights = T * N * (-(-K // 2) + -(-K // 32) + (4 if case["bias"] else 0))
        return {"bytes": weights + R * K * x + R * N * (2 if case["y"] == "bf16" else 4), "flops": 2 * R * K * N}
    R, C = case["rows"], case["classes"] * (0.875 if case["ragged"] else 1.0)
    touched = R * C * ((2 if case["dtype"] == "bf16" else 4) + (1 / 8 if case["masked"] else 0))
    return {"bytes": touched + R * (4 + 12 * case["given"] + 8 * case["top"]), "flops": 6 * R * C}
