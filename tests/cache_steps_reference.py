"""Windowed and tree attention over the paged cache, the weights of its keys, selection and compaction in plain
64-bit torch, on the host, one sequence and head at a time (beside cache_reference.py)."""
from __future__ import annotations

import math

import torch

from cache_reference import BLOCK, D, e4m3


def causal(n, L, tokens=None):
    """[n, L]: which keys the last n tokens of L see."""
    return torch.arange(L) <= torch.arange(L - n, L)[:, None]


def everything(n, L, tokens=None):
    return torch.ones((n, L), dtype=torch.bool)


def window(size, sinks, is_causal):
    def sees(n, L, tokens=None):
        end = torch.arange(L - n + 1, L + 1)[:, None] if is_causal else torch.full((n, 1), L)
        j = torch.arange(L)
        return (j < end) & ((j >= end - size) | (j < sinks))
    return sees


def tree(mask):
    """mask int32 [tokens, words] on the host."""
    def sees(n, L, tokens):
        m = mask[tokens].long() & 0xFFFFFFFF
        out = torch.zeros((n, L), dtype=torch.bool)
        for j in range(L):
            d = j - (L - n)
            if d < 0:
                out[:, j] = True
            elif d // 32 < m.shape[1]:
                out[:, j] = (m[:, d // 32] >> (d % 32)) & 1 == 1
        return out
    return sees


def attend(cache, q, table, q_start, kv_len, sees):
    """[tokens, Hq, d] fp64, a bound on the error of the kernel's result, and {(s, head): (weights [L], bound, bound
    where l is a sum of the scores that become weights too)}.

    The bound of the output is that of cache_reference.attend.  A weight is the sum over rows of p = 2^(s c - m) / l:
    each p is off by its score's error and exp2's (rel below), by l's (at most the largest error of the row's p, whose
    scores may be of the FP8 matrix cores: 2^-15 of sum |q k|, and 2^-18 from the chain of its additions) and by one
    more rounding each of 1 / l and of the product (2^-23); the fp32 sum of up to 2^14 positive terms, 32 at a time in
    parallel, adds at most 2^-15 of itself in a chain of 2^9 additions.  Where up to 32 rows' scores are kept, l is
    their sum, and a weight that of at most 2^6 terms."""
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    weights = {}
    Hq, Hkv = q.shape[1], cache.k.shape[1]
    for s in range(len(kv_len)):
        n, L = q_start[s + 1] - q_start[s], kv_len[s]
        tokens = slice(q_start[s], q_start[s + 1])
        for h in range(Hkv if n else 0):
            k, v = cache.rows(table[s], L, h)
            hidden = ~sees(n, L, tokens)
            total, bound, near = (torch.zeros(L, dtype=torch.float64) for _ in range(3))
            for g in range(Hq // Hkv):
                i = h * (Hq // Hkv) + g
                x = q[tokens, i].double()
                t = x @ k.t() / math.sqrt(D)
                err = (2.0 ** -22 * x.abs().amax(-1, keepdim=True) * k.abs().sum(-1)
                       + 2.0 ** -20 * x.abs() @ k.abs().t()) / math.sqrt(D)
                t = t.masked_fill(hidden, -math.inf)
                m = t.amax(-1, keepdim=True) if L else torch.zeros(n, 1)
                m = torch.where(m == -math.inf, 0.0, m)
                p = torch.exp(t - m)
                l = p.sum(-1, keepdim=True)
                p = torch.where((l > 0) | l.isnan(), p / l, 0.0)
                vv = torch.where(torch.isnan(v), 0.0, v)
                nan = ((~hidden).double() @ torch.isnan(v).double() > 0) if L else torch.zeros(n, D, dtype=bool)
                o = torch.where(nan, math.nan, p @ vv)
                rel = torch.where(hidden, 0.0, 2 * err + 2.0 ** -21 * (torch.where(hidden, 0.0, t.abs()) + m.abs()))
                drift = rel.amax(-1, keepdim=True) if L else torch.zeros(n, 1)
                fp8 = torch.where(hidden, 0.0, 2.0 ** -15 * (x.abs() @ k.abs().t()) / math.sqrt(D))
                sums = drift + (fp8.amax(-1, keepdim=True) if L else torch.zeros(n, 1))
                out[tokens, i] = o
                tol[tokens, i] = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -17 + 2 * drift) * (p @ vv.abs())
                total += p.sum(0)
                bound += (p * (rel + sums + 2.0 ** -18 + 2.0 ** -22)).sum(0)
                near += (p * (rel + drift + 2.0 ** -18 + 2.0 ** -22)).sum(0)
            weights[s, h] = total, bound + 2.0 ** -15 * total, near + 2.0 ** -18 * total
    return out, tol, weights


def weights_of(w, table, length, head):
    """[length] of a sequence's weights w [pages, heads, page_tokens]."""
    t = torch.arange(length)
    return w[table[t // w.shape[2]].long(), head, t % w.shape[2]]


def select(w, table, kv_len, budget, sinks, recent):
    S, H = len(kv_len), w.shape[1]
    kept = torch.full((S, H, budget), -1, dtype=torch.int32)
    for s, L in enumerate(kv_len):
        for h in range(H):
            stay = list(range(L))
            if L > budget:
                x = weights_of(w, table[s], L, h).tolist()
                middle = [(math.isnan(x[j]), 0.0 if math.isnan(x[j]) else -x[j], j) for j in range(sinks, L - recent)]
                stay = sorted(list(range(sinks)) + [j for _, _, j in sorted(middle)[:budget - sinks - recent]]
                              + list(range(L - recent, L)))
            kept[s, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
    return kept, [min(L, budget) for L in kv_len]


def compact(cache, table, out_table, kept, counts, base, w=None):
    """Moves the tokens of `cache` (cache_reference.Cache) and of w [pages, heads, page_tokens]; all that is moved is
    read before any of it is written."""
    P, H, page = cache.k.shape[:3]
    moved = []
    for s, n in enumerate(counts):
        if not 1 <= n <= kept.shape[2] or base[s] < 0 or base[s] + n > out_table.shape[1] * page:
            continue
        for h in range(H):
            row = kept[s, min(h, kept.shape[1] - 1)].tolist()
            for b in range(base[s] // BLOCK, -(-(base[s] + n) // BLOCK)):
                to = int(out_table[s, b * BLOCK // page])
                if not 0 <= to < P:
                    continue
                src, ws = [], []  # (page, place) or None for no such token
                for j in range(b * BLOCK, min((b + 1) * BLOCK, base[s] + n)):
                    t, f = (out_table, j) if j < base[s] else (table, row[j - base[s]])
                    p = int(t[s, f // page]) if 0 <= f < t.shape[1] * page else -1
                    src.append((p, f % page) if 0 <= p < P else None)
                for X, E in ((cache.k, cache.ke), (cache.v, cache.ve)):
                    e = [None if x is None or int(E[x[0], h, x[1] // BLOCK]) == 128 else int(E[x[0], h, x[1] // BLOCK])
                         for x in src]
                    top = max([x for x in e if x is not None], default=-127)
                    y = torch.zeros((BLOCK, D), dtype=torch.float64)
                    for i, x in enumerate(src):
                        y[i] = math.nan if e[i] is None else e4m3(X[x[0], h, x[1]] * 2.0 ** (e[i] - top))
                    moved.append((X, E, to, h, b * BLOCK % page, y, top))
                if w is not None:
                    first = max(base[s] - b * BLOCK, 0)
                    ws = [0.0 if x is None else float(w[x[0], h, x[1]]) for x in src[first:]]
                    moved.append((w, None, to, h, b * BLOCK % page + first, ws, None))
    for X, E, to, h, o, y, top in moved:
        if E is None:
            X[to, h, o:o + len(y)] = torch.tensor(y)
        else:
            X[to, h, o:o + BLOCK] = y
            E[to, h, o // BLOCK] = top
