"""The 8-bit cache's operators in 64 bits, from their definitions, on the CPU (test infrastructure; no code of the package).

A cache is held as numbers: per pool `num` [num_pages, n_kv, 64, dh] float64 (what the codes stand for in units of the
scale) and `scale` [num_pages, n_kv] float64 powers of two."""
import math

import torch

PAGE = 64
LARGEST = {"e4m3": 448.0, "int8": 127.0}
E_MIN, E_MAX = -32, 64


def numbers(codes, fmt):
    """uint8 codes -> the numbers they stand for, by the formats' definitions."""
    c = codes.cpu().to(torch.int64)
    if fmt == "int8":
        return torch.where(c > 127, c - 256, c).double()
    sign, exp, man = c >> 7, (c >> 3) & 15, (c & 7).double()
    mag = torch.where(exp == 0, man * 2.0 ** -9, (1 + man / 8) * torch.exp2((exp - 7).double()))
    mag = torch.where((exp == 15) & (man == 7), math.nan, mag)
    return torch.where(sign == 1, -mag, mag)


def nearest(x, fmt):
    """The format's number nearest to x, ties to even; |x| is at most the largest."""
    if fmt == "int8":
        return torch.round(x)
    _, e = torch.frexp(x)                       # x = m 2^e, 0.5 <= |m| < 1
    step = torch.exp2((e - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def scale_for(largest, fmt):
    """Smallest power of two in range that fits; NaN when nothing does."""
    if not largest <= LARGEST[fmt] * 2.0 ** E_MAX:
        return math.nan
    e = E_MIN
    while largest > LARGEST[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Pool:
    def __init__(self, codes, scale, fmt):
        self.fmt, self.num, self.scale = fmt, numbers(codes, fmt), scale.cpu().double().clone()

    def rows(self, table, length, h):
        """[length, dh] values of one sequence and head."""
        ids = table[:(length + PAGE - 1) // PAGE].long()
        return (self.num[ids, h] * self.scale[ids, h][:, None, None]).flatten(0, 1)[:length]

    def codes_and_scales(self, table, length, h):
        """[length, dh] codes and [length] scales of one sequence and head."""
        ids = table[:(length + PAGE - 1) // PAGE].long()
        return self.num[ids, h].flatten(0, 1)[:length], self.scale[ids, h].repeat_interleave(PAGE)[:length]

    def write(self, table, ctx, x):
        """x [q, n_kv, dh] float64 behind ctx cached tokens."""
        q = x.shape[0]
        for blk in range(ctx // PAGE, (ctx + q + PAGE - 1) // PAGE):
            lo, hi = max(ctx, blk * PAGE), min(ctx + q, blk * PAGE + PAGE)
            page, have = int(table[blk]), lo - blk * PAGE
            for h in range(x.shape[1]):
                part = x[lo - ctx:hi - ctx, h]
                s = scale_for(float(part.abs().max()), self.fmt) if bool(torch.isfinite(part).all()) else math.nan
                held = float(self.scale[page, h])
                if have:
                    s = math.nan if math.isnan(held) else (s if math.isnan(s) else max(s, held))
                if math.isnan(s):
                    self.num[page, h, have:hi - blk * PAGE] = 0.0
                else:
                    if have:
                        self.num[page, h, :have] = nearest(self.num[page, h, :have] * (held / s), self.fmt)
                    self.num[page, h, have:hi - blk * PAGE] = nearest(part / s, self.fmt)
                self.scale[page, h] = s


def attend(kpool, vpool, table, ctx, q_lens, q, w_in=None, window=0):
    """q [tokens, n_q, dh].  Returns o, its error scales (what relative and what absolute errors of the probabilities make
    of it, see check_attend), the largest sum_d |q_d k_d| / sqrt(dh) of every row, and the new weights (list over sequences
    of [n_kv, len])."""
    n_kv = kpool.num.shape[1]
    tokens, n_q, dh = q.shape
    g = n_q // n_kv
    q = q.cpu().double()
    o, rel, sub = (torch.zeros(tokens, n_q, dh, dtype=torch.float64) for _ in range(3))
    big = torch.zeros(tokens, n_q, dtype=torch.float64)
    weights, at = [], 0
    for b, n in enumerate(q_lens):
        full = ctx[b] + n
        w = None if w_in is None else w_in[b, :, :full].cpu().double().clone()
        hidden = torch.arange(full)[None] > (ctx[b] + torch.arange(n))[:, None]
        for h in range(n_kv if n else 0):
            k, v = kpool.rows(table[b], full, h), vpool.rows(table[b], full, h)
            for a in range(h * g, h * g + g):
                x = q[at:at + n, a]
                s = (x @ k.T / math.sqrt(dh)).masked_fill(hidden, -math.inf)
                p = torch.softmax(s, -1)
                o[at:at + n, a], rel[at:at + n, a] = p @ v, p @ v.abs()
                c, sc = vpool.codes_and_scales(table[b], full, h)
                sub[at:at + n, a] = (p * sc).amax(-1, keepdim=True) * ((~hidden).double() @ c.abs())
                big[at:at + n, a] = (x.abs() @ k.abs().T / math.sqrt(dh)).masked_fill(hidden, 0).amax(-1)
                if w is not None:
                    w[h] += p[max(0, n - window) if window else 0:].sum(0)
        weights.append(w)
        at += n
    return o, (rel, sub), big, weights


def check_attend(got, o, mag, big):
    """|error| of every element: the output's rounding to bf16 (2^-8 of the value), P's rounding to fp16 (2^-11 each, so
    2^-11 sum p |v|, and where p times its V scale is so small that fp16 holds it as a denormal number, by 2^-25 of a unit
    that is at most 2^-6 of the largest such product: 2^-31 max(p s) sum |c|, c and s V's codes and scales), and what the
    scores are off in fp32: a product sum of up to 128 terms, at most 2^-17 of
    sum |q k| / sqrt(dh) in all (128 roundings of 2^-24), times log2 e in the exponent; p is off by that much relatively,
    twice with the normalisation.  2^-20 for the exponentials, the sums and the merging factors."""
    got = got.cpu().double()
    rel_p = 2.0 ** -11 + 2 * 2.0 ** -17 * big[..., None] + 2.0 ** -18
    tol = 2.0 ** -8 * o.abs() + rel_p * mag[0] + 2.0 ** -31 * mag[1] + 1e-38
    err = (got - o).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).nan_to_num(1e9).max()):.3g} x the bound"


def check_weights(got, weights, w_in, big_all):
    """Sums of at most 2^-17-scale errors of the scores (see check_attend), exponentials and fp32 adds."""
    for b, w in enumerate(weights):
        g = got[b, :, :w.shape[1]].cpu().double()
        added = w - w_in[b, :, :w.shape[1]].cpu().double()
        tol = (2 * 2.0 ** -17 * big_all + 2.0 ** -17) * added + 2.0 ** -22 * w.abs() + 1e-30
        err = (g - w).abs()
        assert bool((err <= tol).all()), f"sequence {b}: worst {float((err / tol).max()):.3g} x the bound"


def evict(kpool, vpool, table, lens, weights, to_table, budget, sink, recent):
    """Writes the destination pages into the pools; returns kept positions [b][h] and new lengths."""
    n_kv = kpool.num.shape[1]
    kept = []
    for b, n in enumerate(lens):
        per_head = []
        for h in range(n_kv):
            if n <= budget:
                keep = list(range(n))
            else:
                w = weights[b, h, :n].tolist()
                order = sorted(range(sink, n - recent), key=lambda j: (-w[j] if w[j] == w[j] else math.inf, j))
                # (a NaN below every number, -inf included)
                order = [j for j in order if w[j] == w[j]] + [j for j in order if w[j] != w[j]]
                keep = sorted(list(range(sink)) + order[:budget - sink - recent] + list(range(n - recent, n)))
            per_head.append(keep)
            at = torch.tensor(keep, dtype=torch.long)
            for pool in (kpool, vpool):
                src = table[b].long()[at // PAGE]
                x = pool.num[src, h, at % PAGE] * pool.scale[src, h][:, None]
                for lo in range(0, len(keep), PAGE):
                    part = x[lo:lo + PAGE]
                    page = int(to_table[b, lo // PAGE])
                    s = scale_for(float(part.abs().max()), pool.fmt) if not bool(torch.isnan(part).any()) else math.nan
                    pool.num[page, h, :len(part)] = 0.0 if math.isnan(s) else nearest(part / s, pool.fmt)
                    pool.scale[page, h] = s
        kept.append(per_head)
    return kept, [min(n, budget) for n in lens]
