"""What the operators around language models' paged caches are measured on: the write of new tokens into the pages, the attention that reads
them, the handling of the pages themselves, and the choice of the next token.

A pass is one call of one operator (of the pages: a few calls as a server makes them together).  Where `own` is false it is computed in its plain
form, elementary torch operations in 32 bits (the choice of a token in 64: sums of many weights stand next to borders there); where it is true, by the runtime's entry points, on
the same inputs and into buffers that the caller holds.

A cache is [layers, pages, heads, page, head_dim] of keys and [layers, pages, heads, head_dim, page] of values (a feature's tokens side by side), a
table [sequences, width] of page numbers, the lengths of the sequences in tokens and, for every page, by how many sequences it is held.  In 8 bits (kv8) values
are e4m3 with a power of two for every token and head.

The keys of a case
  op        write:  the last tokens of every sequence into its pages
            attend: the last tokens of every sequence attend to all of it, each up to itself
            pages:  fork (drop children, fork parents into them, make room for their next tokens) or turnover (half of the sequences leave, the pages
                    are compacted, others take their place; then the other half)
            sample: a token for every row of logits, from a given random number
  caches    seqs; lo, hi (tokens: spread over lo..hi); page (tokens); kv_heads, head_dim; dtype (bf16, f32: of rows, and of the cache unless kv8)
  attend    q_heads; new (tokens of a sequence that attend: 1..new); window (tokens that one sees; 0: all); mixed (the batch names its sequences, in another order)
  write     before (tokens that are there already: 0..before)
  pages     what; children; layers; room (tokens)
  sample    rows, classes, dtype; top_k (rows draw theirs up to it; 0: none), top_p, min_p (rows draw theirs from it on; 1 or 0: none), hot (temperatures
            drawn around 1, some 0), masked (a bit for each class says whether it is allowed), ragged (rows have class counts of their own)
"""
import math
from types import SimpleNamespace

import torch

own = False
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    attend, write, pages, sample = {"op": "attend"}, {"op": "write"}, {"op": "pages"}, {"op": "sample"}
    return [
        # one request to a small model: latency
        dict(attend, name="attend_one_short", seqs=1, lo=333, hi=333, new=1, q_heads=8, kv_heads=2, head_dim=64, page=16, dtype="bf16", kv8=False, window=0, mixed=False),
        # a step of many tenants' requests of all lengths
        dict(attend, name="attend_step", seqs=64, lo=1, hi=4096, new=1, q_heads=32, kv_heads=8, head_dim=128, page=64, dtype="bf16", kv8=False, window=0, mixed=True),
        # one request with a long document: the cache has to be shared among the whole machine
        dict(attend, name="attend_one_long", seqs=1, lo=131072, hi=131072, new=1, q_heads=32, kv_heads=8, head_dim=128, page=64, dtype="bf16", kv8=False, window=0, mixed=False),
        # a full machine in 8 bits: memory decides
        dict(attend, name="attend_kv8_batch", seqs=32, lo=12289, hi=16384, new=1, q_heads=32, kv_heads=8, head_dim=128, page=64, dtype="bf16", kv8=True, window=0, mixed=False),
        # a few proposed tokens each, a window, sizes that fit no tile, fp32
        dict(attend, name="attend_f32_proposals", seqs=9, lo=3, hi=1531, new=5, q_heads=15, kv_heads=3, head_dim=80, page=32, dtype="f32", kv8=False, window=1000, mixed=True),
        # a token of every request of a step
        dict(write, name="write_step_kv8", seqs=256, lo=1, hi=1, before=4096, kv_heads=8, head_dim=128, page=64, dtype="bf16", kv8=True),
        # prompts of a few tenants
        dict(write, name="write_prompts", seqs=8, lo=1500, hi=4096, before=0, kv_heads=8, head_dim=128, page=64, dtype="bf16", kv8=False),
        # one request answered four times over
        dict(pages, name="pages_fork_one", what="fork", seqs=1, children=4, lo=700, hi=700, room=1, layers=2, page=16, kv_heads=2, head_dim=64, dtype="bf16", kv8=False),
        # a server's requests come and go
        dict(pages, name="pages_turnover", what="turnover", seqs=64, children=0, lo=100, hi=2000, room=0, layers=4, page=32, kv_heads=8, head_dim=128, dtype="bf16", kv8=False),
        # the next token of one request: latency
        dict(sample, name="sample_one_row", rows=1, classes=32768, dtype="f32", top_k=50, top_p=0.9, min_p=0.0, hot=False, masked=False, ragged=False),
        # a step of several tenants, each with its own settings, some with a grammar
        dict(sample, name="sample_step", rows=64, classes=65001, dtype="bf16", top_k=200, top_p=0.8, min_p=0.02, hot=True, masked=True, ragged=True),
        # a full machine, all of the distribution but its tail
        dict(sample, name="sample_many", rows=1024, classes=32768, dtype="f32", top_k=0, top_p=0.95, min_p=0.0, hot=False, masked=False, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(("attend", "attend", "attend", "write", "pages", "sample", "sample"))
        if op == "sample":
            c = {"op": op, "rows": _log_int(rng, 1, 1024), "classes": _log_int(rng, 10, 131072), "dtype": rng.choice(("bf16", "f32")), "top_k": rng.choice((0, 0, 1, 20, 50, 200, 3000)),
                 "top_p": rng.choice((1.0, 1.0, 0.95, 0.8, 0.5)), "min_p": rng.choice((0.0, 0.0, 0.02, 0.1)), "hot": rng.random() < 0.5, "masked": rng.random() < 0.3, "ragged": rng.random() < 0.4}
            if c["rows"] * c["classes"] <= 1024 * 32768:
                return c
            continue
        heads = rng.choice((1, 2, 3, 4, 8))
        c = {"op": op, "seqs": _log_int(rng, 1, 256), "page": rng.choice((16, 32, 64, 128)), "kv_heads": heads, "head_dim": rng.choice((64, 128, 64, 128, 80, 96, 192, 256)),
             "dtype": rng.choice(("bf16", "bf16", "f32")), "kv8": rng.random() < 0.4}
        token = heads * c["head_dim"] * (1 if c["kv8"] else 2 if c["dtype"] == "bf16" else 4)
        if op == "attend":
            c["hi"] = _log_int(rng, 1, 131072)
            c["lo"] = _log_int(rng, 1, c["hi"])
            c.update(new=rng.choice((1, 1, 1, 2, 5, 16)), q_heads=heads * rng.choice((1, 1, 2, 4, 5, 8, 16)), window=rng.choice((0, 0, 0, 500, 4096)), mixed=rng.random() < 0.5)
            # (the plain form holds every sequence as if it were as long as the longest, in 32 bits)
            fits = c["seqs"] * c["hi"] * token <= 32 * 16384 * 1024 and c["seqs"] * c["hi"] * c["q_heads"] * c["new"] <= 32 * 16384 * 32 and c["seqs"] * c["hi"] * heads * c["head_dim"] <= 32 * 16384 * 1024
        elif op == "write":
            c["hi"] = _log_int(rng, 1, 4096)
            c["lo"], c["before"] = _log_int(rng, 1, c["hi"]), rng.choice((0, 100, 4096))
            fits = c["seqs"] * c["hi"] * heads * c["head_dim"] <= 8 * 4096 * 1024 and c["seqs"] * c["before"] * heads * c["head_dim"] <= 256 * 4096 * 1024
        else:
            c["hi"] = _log_int(rng, 16, 4096)
            c["lo"], c["layers"] = _log_int(rng, 1, c["hi"]), rng.choice((1, 2, 4))
            c["what"] = rng.choice(("fork", "turnover"))
            c["children"], c["room"] = (rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 7, 100))) if c["what"] == "fork" else (0, 0)
            held = c["seqs"] * (c["hi"] + c["children"] * (c["page"] + c["room"] + c["page"]))
            fits = c["seqs"] > (c["what"] == "turnover") and held * token * c["layers"] <= 64 * 2000 * 8192
        if fits:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n sizes, spread over lo..hi; one alone gets hi."""
    span = hi - lo + 1
    return [hi - (i * 7919) % span for i in range(n)]


def _pages(tokens, page):
    return -(-tokens // page)


def _sizes(case):
    """(tokens of every sequence when the pass begins, new tokens among them)."""
    n = case["seqs"]
    if case["op"] == "write":
        new = _spread(n, case["lo"], case["hi"])
        return [t + (i * 6007) % (case["before"] + 1) for i, t in enumerate(new)], new
    tokens = _spread(n, case["lo"], case["hi"])
    return tokens, [min(t, 1 + (i * 3) % case["new"] if i else case["new"]) for i, t in enumerate(tokens)] if case["op"] == "attend" else [0] * n


def _cache(case, n_pages, seqs, width):
    """An empty cache; the same tensors either way."""
    L, H, D, T = case.get("layers", 1), case["kv_heads"], case["head_dim"], case["page"]
    if own:
        import paper_1901_06887_amd as mt
        return mt.alloc_kv(n_pages, T, H, D, seqs, width, dtype=mt.MT_KV8 if case["kv8"] else mt.MT_BF16 if case["dtype"] == "bf16" else mt.MT_F32, layers=L,
                           device=torch.device("cuda", torch.cuda.current_device()))
    dt = torch.float8_e4m3fn if case["kv8"] else DTYPES[case["dtype"]]
    new = lambda dt, *shape: torch.empty(*shape, dtype=dt, device="cuda")  # noqa: E731
    scales = (lambda: new(torch.float8_e8m0fnu, L, n_pages, H, T)) if case["kv8"] else lambda: None
    return SimpleNamespace(k=new(dt, L, n_pages, H, T, D), v=new(dt, L, n_pages, H, D, T), k_scales=scales(), v_scales=scales(),
                           table=new(torch.int32, seqs, width).fill_(-1), lengths=new(torch.int32, seqs).zero_(), refs=new(torch.int32, n_pages).zero_())


def _fill(cache, g):
    """Keys and values as a model's layers leave them; in 8 bits with the scales that rows of some 1 to 4 in magnitude get."""
    for x, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        for layer in range(x.shape[0]):
            r = torch.randn(x.shape[1:], generator=g, device="cuda")
            if scales is None:
                x[layer].copy_(r)
            else:
                x[layer].copy_((r * 100.0).clamp(-448, 448))
                scales[layer].view(torch.uint8).copy_(torch.randint(119, 122, scales.shape[1:], generator=g, device="cuda", dtype=torch.uint8))


def _hold(cache, tokens, page, order):
    """Tables, lengths and counts of sequences that hold pages in the given order of numbers."""
    table, at = torch.full(cache.table.shape, -1, dtype=torch.int32), 0
    for s, t in enumerate(tokens):
        n = _pages(t, page)
        table[s, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(cache.refs.shape, dtype=torch.int32)
    refs[order[:at].long()] = 1
    cache.table.copy_(table)
    cache.refs.copy_(refs)
    cache.lengths.copy_(torch.tensor(list(tokens) + [0] * (cache.lengths.shape[0] - len(tokens)), dtype=torch.int32))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed * 1000003 + 17)
    host = torch.Generator().manual_seed(seed * 1000003 + 17)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": case}
    if own:
        import paper_1901_06887_amd as mt
        s["ctx"] = mt.Context(1, 1, 64, 1, 1 << 16, mt.MT_BF16, torch.cuda.current_device())
    if case["op"] == "sample":
        R, C = case["rows"], case["classes"]
        uniform = lambda hi, *shape: torch.randint(hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
        rand = lambda: torch.rand(R, generator=g, device="cuda")  # noqa: E731
        s["logits"] = (2.5 * randn(R, C) + 9.0 * (torch.rand(R, C, generator=g, device="cuda") < 4.0 / C)).to(DTYPES[case["dtype"]])
        s["uniform"] = rand()
        s["temperature"] = torch.where(rand() < 0.1, 0.0, 0.5 + rand()) if case["hot"] else None
        s["top_k"] = 1 + uniform(case["top_k"], R) if case["top_k"] else None
        s["top_p"] = case["top_p"] + (1.0 - case["top_p"]) * rand() if case["top_p"] < 1 else None
        s["min_p"] = case["min_p"] * (0.5 + rand()) if case["min_p"] else None
        s["n"] = (C - uniform(C // 4 + 1, R)).to(torch.int32) if case["ragged"] else None
        s["allowed"] = uniform(1 << 16, R, -(-C // 32)) | (uniform(1 << 15, R, -(-C // 32)) << 16) if case["masked"] else None
        if own:
            s["out"] = mt.alloc_samples(R, C, device=s["logits"].device)
        return s
    tokens, new = _sizes(case)
    n, T = case["seqs"], case["page"]
    held, slots, width = sum(_pages(t, T) for t in tokens), n, max(_pages(t, T) for t in tokens)
    if case["op"] == "pages" and case["what"] == "fork":
        slots, width = n * (1 + case["children"]), _pages(case["hi"] + case["room"], T)
        n_pages = held + n * case["children"] * (1 + _pages(case["room"], T) + 1)
    else:
        n_pages = held + held // 8 + 1
    s["cache"] = cache = _cache(case, n_pages, slots, width)
    _fill(cache, g)
    _hold(cache, tokens, T, torch.randperm(n_pages, generator=host).to(torch.int32))
    if case["op"] == "pages":
        if case["what"] == "fork":
            s["children"] = _ints(range(n, slots))
            s["parents"] = _ints([c // case["children"] for c in range(slots - n)])
            s["room"] = _ints([case["room"]] * (slots - n))
        else:
            s["halves"] = [(_ints(ids), _ints([tokens[i] for i in ids])) for ids in (range(n // 2), range(n // 2, n))]
        return s
    order = torch.randperm(n, generator=host).tolist() if case.get("mixed") else list(range(n))
    counts = [new[i] for i in order]
    rows = sum(counts)
    s["ids"] = _ints(order) if case.get("mixed") else None
    s["new"] = max(counts)
    s["first"] = _ints([sum(counts[:i]) for i in range(n + 1)]) if s["new"] > 1 else None
    dt, H, D = DTYPES[case["dtype"]], case["kv_heads"], case["head_dim"]
    if case["op"] == "write":
        # (as one projection leaves them: keys and values of a row side by side)
        kv = randn(rows, 2 * H * D) * torch.where(torch.rand(2 * H * D, generator=g, device="cuda") < 0.02, 5.0, 1.0)
        s["k"], s["v"] = kv.to(dt).split(H * D, 1)
    else:
        s["q"] = (2.0 * randn(rows, case["q_heads"] * D)).to(dt)
        if own:
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(rows, case["q_heads"], dtype=torch.float32, device="cuda")
            s["scratch"] = mt.alloc_attend(s["ctx"], cache, case["q_heads"], n, max_new=s["new"], max_length=max(tokens))
            s["longest"] = max(tokens)
    return s


# ---- the operators ----------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state, state["case"])


def _own_attend(s, case):
    import paper_1901_06887_amd as mt
    mt.attend(s["ctx"], s["cache"], s["q"], s["out"], seqs=s["ids"], first_row=s["first"], max_new=s["new"], max_length=s["longest"], window=case["window"], lse=s["lse"], scratch=s["scratch"])
    return {"out": s["out"], "lse": s["lse"]}


def _whole(c):
    return {"k": c.k, "v": c.v, "k_scales": c.k_scales, "v_scales": c.v_scales}


def _own_write(s, case):
    import paper_1901_06887_amd as mt
    mt.kv_write(s["ctx"], s["cache"], s["k"], s["v"], first_row=s["first"], max_new=s["new"])
    return _whole(s["cache"])


def _own_pages(s, case):
    import paper_1901_06887_amd as mt
    ctx, c = s["ctx"], s["cache"]
    if case["what"] == "fork":
        mt.kv_free(ctx, c, s["children"])
        mt.kv_fork(ctx, c, s["parents"], s["children"])
        mt.kv_grow(ctx, c, s["room"], seqs=s["children"])
    else:
        for ids, tokens in s["halves"]:
            mt.kv_free(ctx, c, ids)
            mt.kv_compact(ctx, c)
            mt.kv_grow(ctx, c, tokens, seqs=ids)
    return {"table": c.table, "lengths": c.lengths, "refs": c.refs, **_whole(c)}


def _own_sample(s, case):
    import paper_1901_06887_amd as mt
    o = mt.sample(s["ctx"], s["logits"], s["uniform"], s["out"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], n_classes=s["n"], allowed=s["allowed"])
    return {"ids": o.ids, "logprobs": o.logprobs, "kept": o.kept}


def _power(scales):
    return (scales.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)


def _rows(s, cache):
    """Of every row its place in the batch, its place among the rows of its sequence, and the tokens up to it."""
    lengths = cache.lengths if s.get("ids") is None else cache.lengths[s["ids"]]
    if s["first"] is None:
        b = torch.arange(lengths.shape[0], device="cuda")
        return b, torch.zeros_like(b), lengths
    first = s["first"].long()
    r = torch.arange((s["k"] if "k" in s else s["q"]).shape[0], device="cuda")
    b = torch.searchsorted(first, r, right=True) - 1
    return b, r - first[b], lengths[b] - (first[b + 1] - r) + 1


def _plain_attend(s, case):
    c, B, T, H, D = s["cache"], case["seqs"], case["page"], case["kv_heads"], case["head_dim"]
    G, n, scale = case["q_heads"] // case["kv_heads"], s["new"], case["head_dim"] ** -0.5
    table = (c.table if s["ids"] is None else c.table[s["ids"]]).clamp(min=0)
    k, v = (t[0].view(torch.uint8)[table].view(t.dtype).float() if case["kv8"] else t[0][table].float() for t in (c.k, c.v))
    if case["kv8"]:
        k, v = k * _power(c.k_scales)[0][table].unsqueeze(-1), v * _power(c.v_scales)[0][table].unsqueeze(-2)
    k = k.permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    v = v.permute(0, 2, 3, 1, 4).reshape(B, H, D, -1)
    b, j, upto = _rows(s, c)
    q = torch.zeros(B, n, H, G, D, device="cuda")
    q[b, j] = s["q"].float().view(-1, H, G, D)
    last = torch.zeros(B, n, dtype=torch.int32, device="cuda")
    last[b, j] = upto.to(torch.int32)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    x = torch.matmul(q, k.transpose(2, 3)) * scale
    t = torch.arange(k.shape[2], device="cuda")
    sees = t < last.unsqueeze(2)
    if case["window"]:
        sees = sees & (t >= last.unsqueeze(2) - case["window"])
    x = torch.where(sees.repeat_interleave(G, 1).unsqueeze(1), x, -math.inf)
    m = x.amax(3, keepdim=True).clamp(min=-3e38)
    e = torch.exp(x - m)
    total = e.sum(3, keepdim=True)
    out = torch.matmul(e, v.transpose(2, 3)) / torch.where(total > 0, total, 1.0)
    back = lambda y: y.view(B, H, n, G, -1).permute(0, 2, 1, 3, 4)[b, j].reshape(b.shape[0], -1)  # noqa: E731
    return {"out": back(out).to(DTYPES[case["dtype"]]), "lse": back(m + torch.log(total))}


def _in_8_bits(x):
    """e4m3 values and e8m0 scales of [rows, heads, head_dim]: the least power of two for every row and head at which none exceeds 448; 1 for zeros."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, (e - 9 + (m > 0.875).to(e.dtype)).clamp(-126, 127), torch.zeros_like(e))
    q = x * ((127 - e).to(torch.int32) << 23).view(torch.float32).unsqueeze(-1)
    return q.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _plain_write(s, case):
    c, T, H, D = s["cache"], case["page"], case["kv_heads"], case["head_dim"]
    b, _, upto = _rows(s, c)
    at = upto - 1
    page, slot = c.table[b, at // T].long(), (at % T).long()
    for x, to, scales, turned in ((s["k"], c.k, c.k_scales, False), (s["v"], c.v, c.v_scales, True)):
        x, to = x.reshape(-1, H, D), to[0]
        if case["kv8"]:
            x, e = _in_8_bits(x.float())
            to = to.view(torch.uint8)
            scales[0].view(torch.uint8)[page, :, slot] = e
        if turned:
            to[page, :, :, slot] = x
        else:
            to[page, :, slot] = x
    return _whole(c)


def _plain_copy(c, src, dst):
    for x in (c.k, c.v, c.k_scales, c.v_scales):
        if x is not None:
            bits = x.view(torch.uint8)
            bits[:, dst] = bits[:, src]


def _plain_free(c, T, ids):
    table = c.table[ids]
    there = torch.arange(table.shape[1], device="cuda") < ((c.lengths[ids] + T - 1) // T).unsqueeze(1)
    pages = table[there].long()
    c.refs.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    c.table[ids] = -1
    c.lengths[ids] = 0


def _plain_grow(c, T, ids, tokens):
    was = c.lengths[ids]
    now = was + tokens
    have, need = (was + T - 1) // T, (now + T - 1) // T
    fits = need <= c.table.shape[1]
    takes = torch.where(fits, need - have, 0)
    free = torch.nonzero(c.refs == 0).squeeze(1)
    fits = fits & ((takes == 0) | (takes.cumsum(0) <= free.shape[0]))
    i = torch.arange(c.table.shape[1], device="cuda")
    sel = (i >= have.unsqueeze(1)) & (i < need.unsqueeze(1)) & fits.unsqueeze(1)
    table = c.table[ids]
    free = free[:int(sel.sum())]
    table[sel] = free.to(torch.int32)
    c.table[ids] = table
    c.refs[free] = 1
    c.lengths[ids] = torch.where(fits, now, was)


def _plain_fork(c, T, parents, children):
    was, table = c.lengths[parents], c.table[parents]
    full, part = was // T, was % T > 0
    free = torch.nonzero(c.refs == 0).squeeze(1)
    fits = (c.lengths[children] == 0) & (~part | (part.cumsum(0) <= free.shape[0]))
    i = torch.arange(table.shape[1], device="cuda")
    shared = (i < full.unsqueeze(1)) & fits.unsqueeze(1)
    pages = table[shared].long()
    c.refs.index_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
    last = (i == full.unsqueeze(1)) & (part & fits).unsqueeze(1)
    src = table[last].long()
    dst = free[:src.shape[0]]
    c.refs[dst] = 1
    mine = torch.where(shared, table, -1)
    mine[last] = dst.to(torch.int32)
    c.table[children] = mine
    c.lengths[children] = torch.where(fits, was, 0)
    _plain_copy(c, src, dst)


def _plain_compact(c):
    live = int((c.refs > 0).sum())
    src, dst = torch.nonzero(c.refs[live:] > 0).squeeze(1) + live, torch.nonzero(c.refs[:live] == 0).squeeze(1)
    _plain_copy(c, src, dst)
    to = torch.arange(c.refs.shape[0], device="cuda", dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    c.table.copy_(torch.where(c.table >= 0, to[c.table.clamp(min=0)], -1))
    c.refs[dst] = c.refs[src]
    c.refs[src] = 0


def _plain_pages(s, case):
    c, T = s["cache"], case["page"]
    if case["what"] == "fork":
        _plain_free(c, T, s["children"])
        _plain_fork(c, T, s["parents"], s["children"])
        _plain_grow(c, T, s["children"], s["room"])
    else:
        for ids, tokens in s["halves"]:
            _plain_free(c, T, ids)
            _plain_compact(c)
            _plain_grow(c, T, ids, tokens)
    return {"table": c.table, "lengths": c.lengths, "refs": c.refs, **_whole(c)}


def _plain_sample(s, case):
    C, none = case["classes"], -math.inf
    x = s["logits"].float()
    j = torch.arange(C, device=x.device)
    if s["n"] is not None:
        x = torch.where(j < s["n"].unsqueeze(1), x, none)
    if s["allowed"] is not None:
        x = torch.where(((s["allowed"][:, j // 32] >> (j % 32).to(torch.int32)) & 1).bool(), x, none)
    column = lambda key, default: torch.full((x.shape[0], 1), default, dtype=torch.float64, device=x.device) if s[key] is None else s[key].double().unsqueeze(1)  # noqa: E731
    t, top_p, min_p, top_k = column("temperature", 1.0), column("top_p", 1.0), column("min_p", 0.0), column("top_k", 0.0)
    x, ids = torch.sort(x, dim=1, descending=True, stable=True)
    z = (x.double() - x[:, :1].double()) / torch.where(t > 0, t, 1.0)
    w = torch.where((t > 0) | (j == 0), torch.exp(z), 0.0)            # in the order of falling logits
    keep = (x > none) & ((j < top_k) | (top_k <= 0)) & (w >= min_p.clamp(max=1)) & ((t > 0) | (j == 0))
    w = torch.where(keep, w, 0.0)
    sums = w.cumsum(1)
    keep = keep & ((sums - w < top_p * sums[:, -1:]) | (top_p >= 1) | (j == 0))
    w = torch.zeros_like(w).scatter_(1, ids, torch.where(keep, w, 0.0))            # in the order of the classes
    sums = w.cumsum(1)
    total = sums[:, -1:]
    kept = keep.sum(1, dtype=torch.int32)
    last = torch.where(w > 0, j, -1).amax(1, keepdim=True)
    at = torch.minimum((sums <= s["uniform"].double().unsqueeze(1) * total).sum(1, keepdim=True), last)
    logprobs = torch.log(w.gather(1, at.clamp(min=0)) / torch.where(total > 0, total, 1.0))
    return {"ids": at.squeeze(1).to(torch.int32), "logprobs": logprobs.squeeze(1).float(), "kept": kept}


_own = {"attend": _own_attend, "write": _own_write, "pages": _own_pages, "sample": _own_sample}
_plain = {"attend": _plain_attend, "write": _plain_write, "pages": _plain_pages, "sample": _plain_sample}


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits; 8-bit values before their rounding.  Whole numbers are held to be equal and left out here, and pages
    that are only moved."""
    global own
    if case["op"] == "pages":
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"attend": _exact_attend, "write": _exact_write, "sample": _exact_sample}[case["op"]](s, case)


def _exact_attend(s, case):
    c, T, H, D = s["cache"], case["page"], case["kv_heads"], case["head_dim"]
    G, rows = case["q_heads"] // H, s["q"].shape[0]
    first = list(range(rows + 1)) if s["first"] is None else s["first"].tolist()
    out = torch.zeros(rows, H, G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((rows, H, G), -math.inf, dtype=torch.float64, device="cuda")
    scale = lambda e: torch.exp2(e.view(torch.uint8).double() - 127)  # noqa: E731
    for b in range(case["seqs"]):
        slot = b if s["ids"] is None else int(s["ids"][b])
        length = int(c.lengths[slot])
        pages = c.table[slot, :_pages(length, T)].long()
        k, v = (t[0].view(torch.uint8)[pages].view(t.dtype).double() if case["kv8"] else t[0][pages].double() for t in (c.k, c.v))
        if case["kv8"]:
            k, v = k * scale(c.k_scales[0][pages])[..., None], v * scale(c.v_scales[0][pages])[..., None, :]
        k, v = k.transpose(0, 1).reshape(H, -1, D)[:, :length], v.permute(1, 0, 3, 2).reshape(H, -1, D)[:, :length]
        for r in range(first[b], first[b + 1]):
            end = length - (first[b + 1] - 1 - r)
            begin = max(0, end - case["window"]) if case["window"] else 0
            if end <= begin:
                continue
            x = torch.bmm(s["q"][r].double().view(H, G, D), k[:, begin:end].transpose(1, 2).contiguous()) / math.sqrt(D)
            lse[r] = torch.logsumexp(x, 2)
            out[r] = torch.bmm(torch.softmax(x, 2), v[:, begin:end].contiguous())
    return {"out": out.view(rows, -1), "lse": lse.view(rows, -1)}


def _exact_write(s, case):
    c, T, H, D = s["cache"], case["page"], case["kv_heads"], case["head_dim"]
    first = list(range(s["k"].shape[0] + 1)) if s["first"] is None else s["first"].tolist()
    page, slot = [], []
    table, lengths = c.table.cpu(), c.lengths.tolist()
    for b in range(case["seqs"]):
        at = torch.arange(lengths[b] - (first[b + 1] - first[b]), lengths[b])
        page.append(table[b].long()[at // T])
        slot.append(at % T)
    page, slot = torch.cat(page).cuda(), torch.cat(slot).cuda()
    o = {"k": c.k.double(), "v": c.v.double(), "k_scales": None, "v_scales": None}
    for name, x in (("k", s["k"]), ("v", s["v"])):
        x = x.double().reshape(-1, H, D)
        if case["kv8"]:
            most = x.abs().amax(2)
            scale = torch.where(most > 0, torch.exp2(torch.ceil(torch.log2(most / 448.0)).clamp(min=-126)), 1.0)
            x = x / scale[..., None]
            o[name + "_scales"] = (c.k_scales if name == "k" else c.v_scales).to(torch.float32).double()
            o[name + "_scales"][0, page, :, slot] = scale
        if name == "k":
            o[name][0, page, :, slot] = x
        else:
            o[name][0, page, :, :, slot] = x
    return o


def _exact_sample(s, case):
    logprobs = []
    # (a row at a time, by sorted weights and searches among their sums)
    for r in range(case["rows"]):
        x = s["logits"][r].double()
        if case["masked"]:
            bits = s["allowed"][r].view(torch.uint8).unsqueeze(1) >> torch.arange(8, device=x.device, dtype=torch.uint8) & 1
            x = torch.where(bits.flatten()[:case["classes"]].bool(), x, -math.inf)
        if case["ragged"]:
            x = x[:int(s["n"][r])]
        t = float(s["temperature"][r]) if case["hot"] else 1.0
        order = torch.argsort(x, descending=True, stable=True)
        n = int((x > -math.inf).sum())
        if n == 0:
            logprobs.append(torch.full((), -math.inf, dtype=torch.float64, device=x.device))
            continue
        if t == 0.0:
            n = 1
        if case["top_k"]:
            n = min(n, int(s["top_k"][r]))
        p = torch.softmax(x[order[:n]] / (t if t > 0 else 1.0), 0)
        if case["min_p"]:
            n = max(1, int((p / p[0] >= float(s["min_p"][r])).sum()))
            p = p[:n] / p[:n].sum()
        if case["top_p"] < 1:
            n = min(n, 1 + int(torch.searchsorted(p.cumsum(0), float(s["top_p"][r]))))
            p = p[:n] / p[:n].sum()
        by_class, place = torch.sort(order[:n])
        p = p[place]
        at = min(n - 1, int(torch.searchsorted(p.cumsum(0), float(s["uniform"][r]), right=True)))
        logprobs.append(torch.log(p[at]))
    return {"ids": None, "logprobs": torch.stack(logprobs), "kept": None}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    if case["op"] == "sample":
        R, C = case["rows"], case["classes"] * (0.875 if case["ragged"] else 1.0)
        return {"bytes": R * C * ((2 if case["dtype"] == "bf16" else 4) + (1 / 8 if case["masked"] else 0)) + R * 32, "flops": 6 * R * C}
    H, D, T = case["kv_heads"], case["head_dim"], case["page"]
    row, token = (2 if case["dtype"] == "bf16" else 4), 2 * H * (D + 1 if case["kv8"] else D * (2 if case["dtype"] == "bf16" else 4))
    tokens, new = _sizes(case)
    if case["op"] == "write":
        return {"bytes": sum(new) * (2 * H * D * row + token), "flops": 4 * sum(new) * H * D}
    if case["op"] == "attend":
        seen = lambda t: min(t, case["window"]) if case["window"] else t  # noqa: E731
        read = sum(min(t, seen(t) + n - 1) for t, n in zip(tokens, new))
        pairs = sum(seen(t - j) for t, n in zip(tokens, new) for j in range(n))
        return {"bytes": read * token + sum(new) * case["q_heads"] * (2 * D * row + 4), "flops": 4 * pairs * case["q_heads"] * D}
    page = T * token * case["layers"]
    if case["what"] == "fork":
        return {"bytes": 2 * case["children"] * sum(t % T > 0 for t in tokens) * page + 12 * case["children"] * sum(_pages(t, T) for t in tokens), "flops": 0}
    # (each half, compacted, moves down into what the other half left)
    halves = [sum(_pages(t, T) for t in part) for part in (tokens[:len(tokens) // 2], tokens[len(tokens) // 2:])]
    return {"bytes": 2 * 2 * min(halves) * page + 24 * sum(halves), "flops": 0}
