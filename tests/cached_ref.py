"""The operators on a paged cache in 64 bits, for the tests: by loops, on the CPU; and what their results may be off by.

A batch here is plain numbers: rows (m of them), `starts`, `lengths`, `table` (lists), and a pool [page][layer][k|v][kv_head][token][head_dim]."""
import math

import torch

U = 2.0 ** -24   # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def cut(v, lo, hi):
    return min(max(v, lo), hi)


class Batch:
    """what starts, lengths and table come to once they are cut to their ranges"""

    def __init__(self, starts, lengths, table, m, pool_pages, page_tokens):
        self.n, self.m, self.pt, self.n_pages = len(lengths), m, page_tokens, pool_pages
        self.table = [list(map(int, t)) for t in table]
        self.slots = len(self.table[0]) * page_tokens if self.n else 0
        self.row0 = [cut(int(starts[s]), 0, m) for s in range(self.n)]
        self.rows = [cut(int(starts[s + 1]), self.row0[s], m) - self.row0[s] for s in range(self.n)]
        self.length = [cut(int(c), 0, self.slots) for c in lengths]

    def slot(self, s, i):
        return self.length[s] - self.rows[s] + i

    def page(self, s, slot):
        p = self.table[s][slot // self.pt]
        return p if 0 <= p < self.n_pages else None

    def seen(self, s, i, causal):
        """the slots that row i of sequence s sees"""
        at = self.slot(s, i)
        end = 0 if at < 0 else at + 1 if causal else self.length[s]
        return [t for t in range(end) if self.page(s, t) is not None]

    def plane(self, pool, s, slots, layer, which, head):
        return torch.stack([pool[self.page(s, t), layer, which, head, t % self.pt] for t in slots]).double()


def frequencies(rotary, base=10000.0):
    return torch.tensor([base ** (-2 * j / rotary) for j in range(rotary // 2)], dtype=torch.float64)


def turned(x, gain, eps, angle, rotary, interleaved, amplitude):
    """(result, tolerance without the last rounding) of [heads][hd], 64-bit; angle [rotary / 2] or None"""
    x = x.double()
    off = torch.zeros_like(x)
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
        # eight squares in a lane and four additions over lanes, half of it behind the root; mean, eps, root, quotient, two products
        off = 14 * U * x.abs()
    y, tol = x.clone(), off.clone()
    if rotary:
        half = rotary // 2
        first = list(range(0, rotary, 2)) if interleaved else list(range(half))
        second = list(range(1, rotary, 2)) if interleaved else list(range(half, rotary))
        c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
        a, b = x[:, first], x[:, second]
        y[:, first], y[:, second] = a * c - b * s, b * c + a * s
        # sine and cosine: the argument's rounding (0.8 U) and the series (3 U), times amplitude (U); two products and their sum (3 U)
        both = (a.abs() + b.abs()) * abs(amplitude)
        tol[:, first] = tol[:, second] = 8 * U * both + (off[:, first] + off[:, second]) * abs(amplitude)
    return y, tol


def append(q, k, v, pool, b, layer, rotary=0, interleaved=False, freqs=None, amplitude=1.0, q_gain=None, k_gain=None, eps=1e-6, positions=None):
    """(q' and its tolerance, NaN where nothing is written; pool and its tolerance), 64-bit"""
    m, nq, hd = q.shape
    out, tol = torch.full((m, nq, hd), math.nan, dtype=torch.float64), torch.zeros(m, nq, hd, dtype=torch.float64)
    new, new_tol = pool.double(), torch.zeros(pool.shape, dtype=torch.float64)
    for s in range(b.n):
        for i in range(b.rows[s]):
            r, slot = b.row0[s] + i, b.slot(s, i)
            angle = None if not rotary else (slot if positions is None else int(positions[r])) * freqs.double()
            out[r], tol[r] = turned(q[r], q_gain, eps, angle, rotary, interleaved, amplitude)
            if slot >= 0 and b.page(s, slot) is not None:
                at = b.page(s, slot), layer
                key, off = turned(k[r], k_gain, eps, angle, rotary, interleaved, amplitude)
                new[at[0], at[1], 0, :, slot % b.pt], new_tol[at[0], at[1], 0, :, slot % b.pt] = key, off
                new[at[0], at[1], 1, :, slot % b.pt] = v[r].double()
    step = half_step(pool.dtype)
    return out, tol + step * out.abs(), new, new_tol + step * new.abs()


def _scores(q, keys, scale):
    """(scores, what they may be off by) of one head's row: products of bf16 are exact, those of fp32 rounded, then hd sums; the scale"""
    s = keys @ q.double() * scale
    mags = keys.abs() @ q.double().abs() * abs(scale)
    return s, (len(q) + 3) * U * mags


def attend(q, pool, b, layer, scale, causal=True):
    """(out, tolerance, lse, tolerance), NaN where nothing is written, 64-bit"""
    m, nq, hd = q.shape
    group = nq // pool.shape[3]
    out, lse = torch.full((m, nq, hd), math.nan, dtype=torch.float64), torch.full((m, nq), math.nan, dtype=torch.float64)
    tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    bf16 = pool.dtype == torch.bfloat16
    for s in range(b.n):
        everything = [t for t in range(b.length[s]) if b.page(s, t) is not None]
        planes = [[b.plane(pool, s, everything, layer, which, h) if everything else None for h in range(pool.shape[3])] for which in (0, 1)]
        for i in range(b.rows[s]):
            n = len(b.seen(s, i, causal))
            for h in range(nq):
                r = b.row0[s] + i
                if n == 0:
                    out[r, h], lse[r, h] = 0.0, -math.inf
                    continue
                keys, values = planes[0][h // group][:n], planes[1][h // group][:n]
                x, off = _scores(q[r, h], keys, scale)
                top = x.max()
                p = torch.exp(x - top)
                total = p.sum()
                p = p / total
                out[r, h] = p @ values
                # a probability: its score and the maximum, the exponent's rounding (log2 e (s - M), and the exponential's two steps)
                each = off + off.max() + (4 + 2 * (top - x)) * 2 * U
                mags = p @ values.abs()
                # in the numerator and, less the rounding to bf16, in the sum; and both are sums of n + a few rescalings
                tol[r, h] = (p * each) @ values.abs() + mags * ((p * each).sum() + 4 * (n + 16) * U)
                if bf16:
                    tol[r, h] += half_step(torch.bfloat16) * mags
                tol[r, h] += half_step(pool.dtype) * out[r, h].abs()
                lse[r, h] = top + torch.log(total)
                lse_tol[r, h] = (p * each).sum() + off.max() + (n + 16) * 2 * U + 4 * U * (top.abs() + total.log())
    return out, tol, lse, lse_tol


def weigh(q, lse, pool, b, layer, scale, before=None, decay=1.0, causal=True):
    """(weights, tolerance), NaN behind the lengths, 64-bit"""
    nkv, nq = pool.shape[3], q.shape[1]
    group = nq // nkv
    out = torch.full((b.n, nkv, b.slots), math.nan, dtype=torch.float64)
    tol = torch.zeros_like(out)
    for s in range(b.n):
        out[s, :, :b.length[s]] = 0.0 if before is None or decay == 0 else decay * before[s, :, :b.length[s]].double()
        tol[s] = 2 * U * torch.nan_to_num(out[s]).abs()
        every = [t for t in range(b.length[s]) if b.page(s, t) is not None]
        if not every:
            continue
        for h in range(nq):
            keys = b.plane(pool, s, every, layer, 0, h // group)
            for i in range(b.rows[s]):
                seen, r = b.seen(s, i, causal), b.row0[s] + i
                if not seen or lse[r, h] == -math.inf:
                    continue
                n = len(seen)
                x, off = _scores(q[r, h], keys[:n], scale)
                p = torch.exp(x - lse[r, h].double())
                out[s, h // group, seen] += p
                # the difference to lse and the exponential's steps, as above; the sum over rows and heads below
                tol[s, h // group, seen] += p * (off + (4 + 2 * (x - lse[r, h].double()).abs() + lse[r, h].double().abs()) * 2 * U)
        tol[s] += (b.rows[s] * group + 2) * U * torch.nan_to_num(out[s]).abs()
    return out, tol


def choose(weights, length, keep, first, recent):
    """the slots that stay, in order: always the first and the recent ones, then by weight (NaN above all), the lowest slot first"""
    if length <= keep:
        return list(range(length))
    always = [t for t in range(length) if t < first or t >= length - recent]
    rest = [t for t in range(length) if first <= t < length - recent]
    rest.sort(key=lambda t: (0 if math.isnan(weights[t]) else 1, 0.0 if math.isnan(weights[t]) else -weights[t], t))
    return sorted(always + rest[:keep - first - recent])


def evict(pool, b, layer, weights, keep, first, recent, table_out=None):
    """(pool, kept, lengths, weights: NaN where they are left alone)"""
    new, nkv = pool.clone(), pool.shape[3]
    kept = torch.full((b.n, nkv, keep), -1, dtype=torch.int32)
    out = torch.full(weights.shape, math.nan, dtype=torch.float32)
    touched = torch.zeros(weights.shape, dtype=torch.bool)
    for s in range(b.n):
        for h in range(nkv):
            stay = choose(weights[s, h].tolist(), b.length[s], keep, first, recent)
            kept[s, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
            out[s, h, :b.length[s]] = 0.0
            out[s, h, :len(stay)] = weights[s, h, stay]
            touched[s, h, :b.length[s]] = True
            pages = b.table[s] if table_out is None else [int(p) for p in table_out[s]]
            for i, t in enumerate(stay):
                if not 0 <= pages[i // b.pt] < b.n_pages:
                    continue
                for which in (0, 1):
                    src = b.page(s, t)
                    new[pages[i // b.pt], layer, which, h, i % b.pt] = 0 if src is None else pool[src, layer, which, h, t % b.pt]
    return new, kept, torch.tensor([min(c, keep) for c in b.length], dtype=torch.int32), out, touched
