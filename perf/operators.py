"""Operators on a paged KV cache held in 8 bits, in their plain form and as calls of the package.

The cache.  Pages of 64 tokens, [num_pages][n_kv][64][head_dim] codes for K and for V, and one scale for each page and
KV head.  A code c of a page with scale s stands for c * s: c is an e4m3 number (largest 448) or an integer in
[-127, 127].  Scales are powers of two, s = 2^e with the smallest e in [-32, 64] for which every row of the page fits
(largest magnitude <= 448 s, or 127 s), so that scaling is exact and a code is ONE rounding (nearest, ties to even).

append   writes the K and V rows of new tokens behind the cached ones.  Where a page already holds rows, its exponent is
         the larger of the one it has and the one the new rows need; the rows it holds are rounded again at that scale.
attend   o = sum_j softmax_j(q k_j / sqrt(head_dim)) v_j over the cached and the new tokens (causal), for one new token a
         sequence or for chunks; optionally weights_out = weights_in + the attention weight that every key received
         from the last `window` queries of its sequence (0: all), summed over the query heads of the KV head.
evict    keeps min(len, budget) tokens of every (sequence, KV head): the first `sink`, the last `recent` and those with
         the largest accumulated weight in between (ties: the lower position), in their order, copied into other pages
         whose scales are made anew from the kept rows.
"""
import math
import random

import torch

own = False

PAGE = 64
LARGEST = {"e4m3": 448.0, "int8": 127.0}
E_MIN, E_MAX = -32, 64


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one request writes its new token: a chat turn on an idle server, latency counts
        _append("append_step_1", "e4m3", 8, 128, 1, 130, 130, 0, 0),
        # a full decode batch writes one token a sequence
        _append("append_step_64", "int8", 4, 128, 64, 64, 1024, 0, 0),
        # four whole prompts of 4096 tokens (the prefill workload of the benchmark)
        _append("append_prompts", "e4m3", 4, 128, 4, 0, 0, 4096, 4096),
        # a mixed batch: prompt chunks of odd lengths behind odd contexts, the narrow heads of the 1B layer
        _append("append_ragged", "int8", 8, 96, 13, 0, 700, 1, 900),
        # one request generates over a short context: latency counts
        _attend("attend_step_1", "e4m3", 16, 4, 128, 1, 777, 777, 0, 0),
        # the decode workload of the benchmark: 64 sequences of 4k to 16k tokens
        _attend("attend_step_64", "e4m3", 16, 4, 128, 64, 4096, 16384, 0, 0),
        # two long documents, the wide layer of the 16-layer stack
        _attend("attend_step_long", "int8", 32, 8, 128, 2, 60000, 65536, 0, 0),
        # a decode batch that keeps the accumulated weights for a later eviction
        _attend("attend_step_weights", "e4m3", 16, 8, 128, 16, 2000, 8000, 0, 0, weights=True),
        # four whole prompts, causal (the prefill workload of the benchmark)
        _attend("attend_prompts", "e4m3", 16, 4, 128, 4, 0, 0, 4096, 4096),
        # prompt chunks over long contexts whose last 32 queries vote on what to keep
        _attend("attend_chunks_weights", "int8", 8, 4, 64, 3, 3000, 16000, 300, 600, weights=True, window=32),
        # one sequence is cut to its budget
        _evict("evict_1", "int8", 4, 128, 1, 1500, 1500, 512, 4, 128),
        # a memory-bound server cuts a whole batch at once
        _evict("evict_32", "e4m3", 8, 128, 32, 4000, 9000, 2048, 4, 256),
    ]


def _append(name, fmt, n_kv, dh, seqs, ctx_lo, ctx_hi, q_lo, q_hi):
    return dict(name=name, op="append", fmt=fmt, n_kv=n_kv, dh=dh, seqs=seqs, ctx_lo=ctx_lo, ctx_hi=ctx_hi, q_lo=q_lo,
                q_hi=q_hi)


def _attend(name, fmt, n_q, n_kv, dh, seqs, ctx_lo, ctx_hi, q_lo, q_hi, weights=False, window=0):
    return dict(name=name, op="attend", fmt=fmt, n_q=n_q, n_kv=n_kv, dh=dh, seqs=seqs, ctx_lo=ctx_lo, ctx_hi=ctx_hi,
                q_lo=q_lo, q_hi=q_hi, weights=weights, window=window)


def _evict(name, fmt, n_kv, dh, seqs, ctx_lo, ctx_hi, budget, sink, recent):
    return dict(name=name, op="evict", fmt=fmt, n_kv=n_kv, dh=dh, seqs=seqs, ctx_lo=ctx_lo, ctx_hi=ctx_hi, budget=budget,
                sink=sink, recent=recent)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    fmt, dh = rng.choice(["e4m3", "int8"]), rng.choice([64, 96, 128])
    n_kv = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["append_step", "append_chunk", "attend_step", "attend_step", "attend_chunk", "attend_chunk", "evict"])
    if kind == "append_step":
        ctx = _log(rng, 1, 1024)
        c = _append("", fmt, n_kv, dh, _log(rng, 1, 200), ctx // 2, ctx, 0, 0)
    elif kind == "append_chunk":
        q = _log(rng, 2, 4096)
        c = _append("", fmt, n_kv, dh, max(1, min(_log(rng, 1, 16), 8192 // q)), 0, _log(rng, 1, 700), max(1, q // 3), q)
    elif kind == "evict":
        ctx, budget = _log(rng, 40, 9000), _log(rng, 40, 2048)
        sink = min(rng.choice([0, 1, 4, 65]), budget)
        c = _evict("", fmt, n_kv, dh, _log(rng, 1, 24), ctx // 2, ctx, budget, sink, rng.randint(0, min(256, budget - sink)))
    else:
        g = rng.choice([1, 2, 4, 8, 16])
        while g * n_kv * dh % 128 or g * n_kv > 64:
            g = rng.choice([1, 2, 4, 8, 16])
        weights = rng.random() < 0.4
        if kind == "attend_step":
            ctx = _log(rng, 1, 65536)
            seqs = max(1, min(_log(rng, 1, 64), 260000 // (ctx * max(1, g // 4))))
            c = _attend("", fmt, g * n_kv, n_kv, dh, seqs, ctx // 2, ctx, 0, 0, weights)
        else:
            q, ctx = _log(rng, 2, 2048), _log(rng, 1, 16384)
            while q * (ctx + q) * g * n_kv * dh > 4 * 4096 * 2048 * 16 * 128:       # the cost of attend_prompts
                q, ctx = q // 2 + 1, ctx // 2 + 1
            most = 4 * 4096 * 2048 * 16 * 128 // (q * (ctx + q) * g * n_kv * dh)
            c = _attend("", fmt, g * n_kv, n_kv, dh, min(_log(rng, 1, 8), most), ctx // 2, ctx, max(1, q // 2), q, weights,
                        rng.choice([1, 16, 32] if q > 128 else [0, 1, 32]))
    del c["name"]
    return c


def lengths(case):
    """Context and chunk lengths of the case's sequences: spread over the given ranges, the largest among them."""
    r = random.Random(case["seqs"] * 1000003 + case["ctx_hi"] * 31 + case.get("q_hi", 0))
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    ctx[r.randrange(len(ctx))] = case["ctx_hi"]
    q_hi = case.get("q_hi", 0)
    q = [r.randint(case["q_lo"], q_hi) for _ in ctx] if q_hi else [1] * len(ctx)
    if q_hi:
        q[r.randrange(len(q))] = q_hi
    return ctx, q


def work(case):
    ctx, q = lengths(case)
    n_kv, dh = case["n_kv"], case["dh"]
    if case["op"] == "append":
        return {"bytes": sum(q) * n_kv * dh * (4 + 2), "flops": 0}
    if case["op"] == "evict":
        kept = sum(min(c, case["budget"]) for c in ctx) * n_kv
        return {"bytes": sum(ctx) * n_kv * 4 + kept * (4 * dh + 4 + 4), "flops": 0}
    full = sum(c + n for c, n in zip(ctx, q))
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, q))
    moved = full * n_kv * 2 * dh + sum(q) * case["n_q"] * dh * 4 + (full * n_kv * 8 if case["weights"] else 0)
    return {"bytes": moved, "flops": 4 * dh * case["n_q"] * pairs}


# ------------------------------------------------------------------------------------------------------- the inputs
class _Shape:
    """What the package reads of a layer's description to plan these operators."""

    def __init__(self, case):
        self.n_kv_heads, self.head_dim, self.page_size = case["n_kv"], case["dh"], PAGE
        self.n_q_heads = case.get("n_q", case["n_kv"])


def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def prepare(case, seed):
    ctx, q = lengths(case)
    n, n_kv, dh = case["seqs"], case["n_kv"], case["dh"]
    dev = torch.device("cuda")
    gen = torch.Generator(dev).manual_seed(seed)
    decode = case["op"] != "evict" and not case["q_hi"]
    evict = case["op"] == "evict"
    total = [c if evict else c + m for c, m in zip(ctx, q)]
    width = max(1, max(_pages_of(t) for t in total))
    dst_width = _pages_of(case["budget"]) if evict else 0
    used = [_pages_of(t) for t in total]
    num_pages = max(1, sum(used) + n * dst_width)
    ids = torch.randperm(num_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros(n, width, dtype=torch.int32, device=dev)
    at = 0
    for b, m in enumerate(used):
        table[b, :m] = ids[at:at + m]
        at += m
    s = dict(case=dict(case), decode=decode, block_table=table, n_tokens=sum(q), max_q_len=max(q),
             context_lens=torch.tensor(ctx, dtype=torch.int32, device=dev),
             q_lens=None if decode or evict else torch.tensor(q, dtype=torch.int32, device=dev))

    def pool():
        shape = (num_pages, n_kv, PAGE, dh)
        exps = torch.randint(-1, 2, (num_pages, n_kv), generator=gen, device=dev)
        if case["fmt"] == "e4m3":       # rows of standard deviation 1/2, 1 or 2
            codes = torch.empty(shape, dtype=torch.uint8, device=dev)
            for lo in range(0, num_pages, 4096):
                part = torch.randn((min(4096, num_pages - lo),) + shape[1:], generator=gen, device=dev)
                codes[lo:lo + 4096] = (part * 64).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            return codes, torch.exp2((exps - 6).float())
        codes = torch.empty(shape, dtype=torch.uint8, device=dev)
        for lo in range(0, num_pages, 4096):
            part = torch.randn((min(4096, num_pages - lo),) + shape[1:], generator=gen, device=dev)
            codes[lo:lo + 4096] = (part * 32).clamp_(-127, 127).round_().to(torch.int8).view(torch.uint8)
        return codes, torch.exp2((exps - 5).float())

    s["k_pages"], s["k_scales"] = pool()
    s["v_pages"], s["v_scales"] = pool()
    if case["op"] == "append":
        s["k"] = torch.randn(sum(q), n_kv, dh, generator=gen, device=dev).to(torch.bfloat16)
        s["v"] = torch.randn(sum(q), n_kv, dh, generator=gen, device=dev).to(torch.bfloat16)
    elif case["op"] == "attend":
        s["q"] = torch.randn(sum(q), case["n_q"], dh, generator=gen, device=dev).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        if case["weights"]:
            s["weights_in"] = torch.rand(n, n_kv, width * PAGE, generator=gen, device=dev)
            s["weights_out"] = torch.zeros(n, n_kv, width * PAGE, device=dev)
    else:
        s["dst_table"] = ids[at:at + n * dst_width].view(n, dst_width).contiguous()
        # accumulated weights fall off like 1 / rank in a shuffled order, with equal ones among them
        w = 1.0 / (1.0 + torch.rand(n, n_kv, width * PAGE, generator=gen, device=dev) * 4096).floor()
        s["weights_in"] = w
        s["weights_out"] = torch.zeros(n, n_kv, dst_width * PAGE, device=dev)
        s["kept"] = torch.full((n, n_kv, case["budget"]), -1, dtype=torch.int32, device=dev)
        s["new_lens"] = torch.zeros(n, dtype=torch.int32, device=dev)
    if own:
        from paper_2605_06206_b200 import cache8
        s["ops"] = cache8.CacheOps(_Shape(case), case["fmt"], max_tokens=sum(q), max_seqs=n, max_context=width * PAGE)
        s["cache"] = cache8.Paged8(s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], table, s["context_lens"], s["q_lens"])
    return s


# ------------------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "evict": _own_evict}[op](state)
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[op](state)


def _held(s):
    """The cache as the numbers its codes stand for, in units of the pages' scales, and the scales."""
    t = torch.float8_e4m3fn if s["case"]["fmt"] == "e4m3" else torch.int8
    return dict(k=s["k_pages"].view(t), v=s["v_pages"].view(t), k_scales=s["k_scales"], v_scales=s["v_scales"])


def _own_append(s):
    s["ops"].append(s["k"], s["v"], s["cache"], max_q_len=s["max_q_len"])
    return _held(s)


def _own_attend(s):
    s["ops"].attend(s["q"], s["cache"], out=s["out"], max_q_len=s["max_q_len"], weights_in=s.get("weights_in"),
                    weights_out=s.get("weights_out"), window=s["case"]["window"])
    return dict(o=s["out"], weights=s.get("weights_out"))


def _own_evict(s):
    c = s["case"]
    s["ops"].evict(s["cache"], s["weights_in"], s["dst_table"], c["budget"], c["sink"], c["recent"], s["new_lens"], s["kept"],
                   s["weights_out"])
    return dict(_held(s), new_lens=s["new_lens"], kept=s["kept"], weights=s["weights_out"])


# ---- plain forms
def _decode(codes, fmt):
    return codes.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float()


def _encode(x, fmt):
    if fmt == "e4m3":
        return x.to(torch.float8_e4m3fn).view(torch.uint8)
    return x.round().to(torch.int8).view(torch.uint8)


def _exponent(largest, fmt):
    """The smallest e in [E_MIN, E_MAX] with largest <= LARGEST * 2^e."""
    m, x = torch.frexp(largest)
    mq, xq = math.frexp(LARGEST[fmt])
    e = (x - xq + (m > mq)).clamp(E_MIN, E_MAX)
    return torch.where(largest > 0, e, E_MIN)


def _plain_append(s):
    c, table = s["case"], s["block_table"].long()
    ctx = s["context_lens"].long()
    q = torch.ones_like(ctx) if s["q_lens"] is None else s["q_lens"].long()
    start = q.cumsum(0) - q
    n_blocks = (s["max_q_len"] + 126) // PAGE
    blk = ctx[:, None] // PAGE + torch.arange(n_blocks, device=ctx.device)              # [n, n_blocks]
    at_seq, at_blk = torch.nonzero(blk * PAGE < (ctx + q)[:, None], as_tuple=True)
    blk, ctx, q, start = blk[at_seq, at_blk], ctx[at_seq], q[at_seq], start[at_seq]
    page = table[at_seq, blk]
    pos = blk[:, None] * PAGE + torch.arange(PAGE, device=ctx.device)                   # [m, 64]
    old = pos < ctx[:, None]
    new = ~old & (pos < (ctx + q)[:, None])
    token = torch.where(new, start[:, None] + pos - ctx[:, None], 0)
    for rows, pages, scales in ((s["k"], s["k_pages"], s["k_scales"]), (s["v"], s["v_pages"], s["v_scales"])):
        x = rows.float()[token].transpose(1, 2)                                         # [m, n_kv, 64, dh]
        x = torch.where(new[:, None, :, None], x, 0)
        e = _exponent(x.abs().amax((2, 3)), c["fmt"])
        held = scales[page]                                                             # [m, n_kv]
        scale = torch.where(old.any(1)[:, None], torch.maximum(held, torch.exp2(e.float())), torch.exp2(e.float()))
        was = pages[page]
        again = _encode(_decode(was, c["fmt"]) * (held / scale)[:, :, None, None], c["fmt"])
        codes = torch.where(old[:, None, :, None], again, was)
        pages[page] = torch.where(new[:, None, :, None], _encode(x / scale[:, :, None, None], c["fmt"]), codes)
        scales[page] = scale
    return _held(s)


def _plain_rows(pages, scales, table, fmt):
    """[n, n_kv, width * 64, dh] values of the sequences' pages."""
    x = _decode(pages[table], fmt) * scales[table][:, :, :, None, None]
    n, w, h, p, d = x.shape
    return x.transpose(1, 2).reshape(n, h, w * p, d)


def _plain_attend(s):
    c, table = s["case"], s["block_table"].long()
    n, n_q, n_kv, dh = c["seqs"], c["n_q"], c["n_kv"], c["dh"]
    ctx = s["context_lens"].long()
    qn = torch.ones_like(ctx) if s["q_lens"] is None else s["q_lens"].long()
    start = qn.cumsum(0) - qn
    m = s["max_q_len"]
    i = torch.arange(m, device=ctx.device)
    there = i < qn[:, None]                                                             # [n, m]
    token = torch.where(there, start[:, None] + i, 0)
    k = _plain_rows(s["k_pages"], s["k_scales"], table, c["fmt"])
    v = _plain_rows(s["v_pages"], s["v_scales"], table, c["fmt"])
    q = s["q"].float()[token].view(n, m, n_kv, n_q // n_kv, dh).permute(0, 2, 3, 1, 4)  # [n, n_kv, g, m, dh]
    j = torch.arange(k.shape[2], device=ctx.device)
    seen = j <= (ctx[:, None] + i)[:, :, None]                                          # [n, m, keys]
    x = q @ k[:, :, None].transpose(-1, -2) / math.sqrt(dh)
    x = torch.where(seen[:, None, None], x, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True))
    p = x / x.sum(-1, keepdim=True)
    # (keys behind a sequence's last one may hold anything)
    v = torch.where((j < (ctx + qn)[:, None])[:, None, :, None], v, 0)
    o = (p @ v[:, :, None]).permute(0, 3, 1, 2, 4).reshape(n, m, n_q, dh)
    at = torch.nonzero(there, as_tuple=True)
    s["out"][token[at]] = o[at].to(torch.bfloat16)
    if c["weights"]:
        votes = there & (i >= (qn - (c["window"] or m))[:, None])
        w = (p * votes[:, None, None, :, None]).sum((2, 3))                             # [n, n_kv, keys]
        real = (j < (ctx + qn)[:, None])[:, None]
        s["weights_out"][:] = torch.where(real, s["weights_in"] + w, s["weights_out"])
    return dict(o=s["out"], weights=s.get("weights_out"))


def _plain_evict(s):
    c, table, to = s["case"], s["block_table"].long(), s["dst_table"].long()
    n, n_kv, budget = c["seqs"], c["n_kv"], c["budget"]
    lens = s["context_lens"].long()
    new = lens.clamp(max=budget)
    j = torch.arange(s["weights_in"].shape[2], device=lens.device)
    real = j < lens[:, None]
    always = (j < c["sink"]) | (j >= (lens - c["recent"])[:, None]) | (lens <= budget)[:, None]
    key = torch.where(always[:, None], math.inf, s["weights_in"])
    key = torch.where(real[:, None], key, -math.inf)
    best = key.sort(dim=-1, descending=True, stable=True).indices[:, :, :budget]
    taken = torch.arange(best.shape[2], device=lens.device) < new[:, None, None]
    kept = torch.where(taken, best, j.numel()).sort(-1).values                          # ascending, the rest last
    taken = taken.expand_as(kept)
    kept = torch.where(taken, kept, 0)
    wide = best.shape[2]
    s["kept"][:, :, :wide] = torch.where(taken, kept, s["kept"][:, :, :wide]).int()
    s["new_lens"][:] = new.int()
    s["weights_out"][:, :, :wide] = torch.where(taken, s["weights_in"].gather(2, kept), s["weights_out"][:, :, :wide])
    # rows of the destination pages, [n, n_kv, blocks, 64]; blocks without a kept row are left as they are
    blocks = (wide + PAGE - 1) // PAGE
    pad = blocks * PAGE - wide
    kept = torch.nn.functional.pad(kept, (0, pad)).view(n, n_kv, blocks, PAGE)
    taken = torch.nn.functional.pad(taken, (0, pad)).view(n, n_kv, blocks, PAGE)
    b, h = torch.arange(n, device=lens.device)[:, None, None, None], torch.arange(n_kv, device=lens.device)[None, :, None, None]
    src = table[b, kept // PAGE]
    at = torch.nonzero(taken.any(-1), as_tuple=True)                                    # (sequence, head, block)
    page = to[at[0], at[2]]
    for pages, scales in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])):
        x = _decode(pages[src, h, kept % PAGE], c["fmt"]) * scales[src, h][..., None]
        x = torch.where(taken[..., None], x, 0)[at]                                     # [m, 64, dh]
        scale = torch.exp2(_exponent(x.abs().amax((1, 2)), c["fmt"]).float())
        pages[page, at[1]] = torch.where(taken[at][..., None], _encode(x / scale[:, None, None], c["fmt"]), pages[page, at[1]])
        scales[page, at[1]] = scale
    return dict(_held(s), new_lens=s["new_lens"], kept=s["kept"], weights=s["weights_out"])


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    ctx, q = lengths(case)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](s, case, ctx, q)


def _numbers(codes, fmt):
    """What codes stand for, by the formats' definitions."""
    c = codes.to(torch.int64)
    if fmt == "int8":
        return torch.where(c > 127, c - 256, c).double()
    sign, exp, man = c >> 7, (c >> 3) & 15, (c & 7).double()
    mag = torch.where(exp == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * torch.exp2((exp - 7).double()))
    return torch.where(sign == 1, -mag, mag)


def _nearest(x, fmt):
    """The format's number nearest to x (|x| <= its largest), ties to even."""
    if fmt == "int8":
        return torch.round(x)
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(min=-6)
    e = torch.where(x.abs() < torch.exp2(e), e - 1, e).clamp(min=-6)
    e = torch.where(x.abs() >= torch.exp2(e + 1), e + 1, e)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _smallest_scale(largest, fmt):
    e = E_MIN
    while e < E_MAX and largest > LARGEST[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def _exact_append(s, case, ctx, q):
    fmt, table, out, at = case["fmt"], s["block_table"].tolist(), {}, 0
    for rows, pages, scales, name in ((s["k"], s["k_pages"], s["k_scales"], "k"), (s["v"], s["v_pages"], s["v_scales"], "v")):
        held, sc = _numbers(pages, fmt), scales.double()
        rows, at = rows.double(), 0
        for b in range(len(ctx)):
            for blk in range(ctx[b] // PAGE, (ctx[b] + q[b] + PAGE - 1) // PAGE):
                lo, hi = max(ctx[b], blk * PAGE), min(ctx[b] + q[b], blk * PAGE + PAGE)
                page, have = table[b][blk], lo - blk * PAGE
                x = rows[at + lo - ctx[b]:at + hi - ctx[b]].transpose(0, 1)              # [n_kv, rows, dh]
                need = torch.tensor([_smallest_scale(v, fmt) for v in x.abs().amax((1, 2)).tolist()], dtype=torch.float64,
                                    device=x.device)
                new = torch.maximum(need, sc[page]) if have else need
                held[page, :, :have] = _nearest(held[page, :, :have] * (sc[page] / new)[:, None, None], fmt)
                held[page, :, have:hi - blk * PAGE] = _nearest(x / new[:, None, None], fmt)
                sc[page] = new
            at += q[b]
        out[name], out[name + "_scales"] = held, sc
    return out


def _exact_attend(s, case, ctx, q):
    fmt, n_kv, g = case["fmt"], case["n_kv"], case["n_q"] // case["n_kv"]
    if sum(a * b for a, b in zip([c + m for c, m in zip(ctx, q)], q)) * case["n_q"] * case["dh"] > 4e12:
        return None
    o = torch.zeros(sum(q), case["n_q"], case["dh"], dtype=torch.float64, device=s["q"].device)
    w = s["weights_out"].double() if case["weights"] else None
    at = 0
    for b in range(len(ctx)):
        full = ctx[b] + q[b]
        ids = s["block_table"][b, :_pages_of(full)].long()
        pos = ctx[b] + torch.arange(q[b], device=o.device)
        hidden = torch.arange(full, device=o.device)[None] > pos[:, None]
        for h in range(n_kv):
            k = (_numbers(s["k_pages"][ids, h], fmt) * s["k_scales"][ids, h].double()[:, None, None]).flatten(0, 1)[:full]
            v = (_numbers(s["v_pages"][ids, h], fmt) * s["v_scales"][ids, h].double()[:, None, None]).flatten(0, 1)[:full]
            got = torch.zeros(full, dtype=torch.float64, device=o.device)
            for a in range(h * g, h * g + g):
                x = (s["q"][at:at + q[b], a].double() @ k.T) * case["dh"] ** -0.5
                p = torch.softmax(x.masked_fill_(hidden, -math.inf), -1)
                o[at:at + q[b], a] = p @ v
                if w is not None:
                    got += p[max(0, q[b] - case["window"]) if case["window"] else 0:].sum(0)
            if w is not None:
                w[b, h, :full] = s["weights_in"][b, h, :full].double() + got
        at += q[b]
    return dict(o=o, weights=w)


def _exact_evict(s, case, ctx, q):
    fmt, budget = case["fmt"], case["budget"]
    kept, lens, w = s["kept"].clone(), s["new_lens"].clone(), s["weights_out"].double()
    held = {n: (_numbers(s[n + "_pages"], fmt), s[n + "_scales"].double()) for n in ("k", "v")}
    for b, n in enumerate(ctx):
        lens[b] = min(n, budget)
        for h in range(case["n_kv"]):
            if n <= budget:
                keep = list(range(n))
            else:
                x = s["weights_in"][b, h, :n].tolist()
                mid = sorted(range(case["sink"], n - case["recent"]), key=lambda j: (-x[j], j))
                keep = sorted(list(range(case["sink"])) + mid[:budget - case["sink"] - case["recent"]] + list(range(n - case["recent"], n)))
            at = torch.tensor(keep, dtype=torch.long, device=w.device)
            kept[b, h, :len(keep)] = at.int()
            w[b, h, :len(keep)] = s["weights_in"][b, h, at].double()
            src = s["block_table"][b].long()[at // PAGE]
            for num, sc in held.values():
                x = num[src, h, at % PAGE] * sc[src, h][:, None]
                for lo in range(0, len(keep), PAGE):
                    part = x[lo:lo + PAGE]
                    scale = _smallest_scale(float(part.abs().max()), fmt)
                    page = int(s["dst_table"][b, lo // PAGE])
                    num[page, h, :len(part)] = _nearest(part / scale, fmt)
                    sc[page, h] = scale
    return dict(k=held["k"][0], v=held["v"][0], k_scales=held["k"][1], v_scales=held["v"][1], new_lens=lens, kept=kept, weights=w)
