"""The operators around the paged cache in plain 64-bit torch, on the host, one
sequence and head at a time."""
from __future__ import annotations

import math

import torch

D = 128
BLOCK = 32


def turned(x, w, eps, cos, sin, pairs):
    """x [..., d] normed and rotated by cos, sin [..., rot / 2] in fp64, and the magnitude that its rounding
    errors are relative to."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    size = x.abs()
    if cos is not None:
        half = cos.shape[-1]
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if pairs == "interleaved" else (i, i + half)
        y, z = x.clone(), size.clone()
        c, s = cos.double(), sin.double()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        z[..., a] = z[..., b] = size[..., a] + size[..., b]
        x, size = y, z
    return x, size


def tables(rows, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(rows, dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def e4m3(y):
    """Nearest E4M3 value (ties to even) of |y| <= 448; NaN stays."""
    m = y.abs().clamp(min=2.0 ** -6)
    e = torch.frexp(m)[1].double() - 1
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def exponent(x):
    """The smallest e >= -127 with max |x| <= 448 * 2^e over the finite values of x."""
    m = float(torch.where(torch.isfinite(x), x.abs(), 0.0).max())
    e = -127
    while m > 448 * 2.0 ** e:
        e += 1
    return e


class Cache:
    """A paged cache as values: K, V [pages, heads, page_tokens, d] (codes without their scale) and exponents
    [pages, heads, blocks]."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        P, H, n = k_scales.shape
        f = lambda t: t.cpu().view(torch.float8_e4m3fn).double()  # noqa: E731
        self.k = f(k_codes).transpose(3, 4).reshape(P, H, n * BLOCK, D).clone()
        self.v = f(v_codes).transpose(3, 4).reshape(P, H, n * BLOCK, D).clone()
        self.ke, self.ve = k_scales.cpu().int() - 127, v_scales.cpu().int() - 127
        self.page = n * BLOCK

    def rows(self, table, length, head):
        """Keys and values [length, d] of a sequence's head."""
        t = torch.arange(length)
        p, o = table[t // self.page].long(), t % self.page
        s = lambda x, e: x[p, head, o] * torch.exp2(e[p, head, o // BLOCK].double())[:, None]  # noqa: E731
        return s(self.k, self.ke), s(self.v, self.ve)


def append(cache, k, v, table, q_start, kv_len):
    """Appends k, v [tokens, heads, d] (fp64, k turned already)."""
    for s in range(len(kv_len)):
        n, L = q_start[s + 1] - q_start[s], kv_len[s]
        for b in range(max(L - n, 0) // BLOCK, -(-L // BLOCK)):
            p, o = int(table[s, b * BLOCK // cache.page]), b * BLOCK % cache.page
            lo, hi = max(L - n, 0, b * BLOCK), min(L, (b + 1) * BLOCK)
            if lo >= hi or not 0 <= p < cache.k.shape[0]:
                continue
            rows = slice(q_start[s] + lo - (L - n), q_start[s] + hi - (L - n))
            for h in range(cache.k.shape[1]):
                for X, E, x in ((cache.k, cache.ke, k), (cache.v, cache.ve, v)):
                    new = x[rows, h]
                    e, was = exponent(new), int(E[p, h, o // BLOCK])
                    if lo > b * BLOCK:
                        e = max(e, was)
                        old = X[p, h, o:o + lo - b * BLOCK]
                        old.copy_(e4m3(old * 2.0 ** (was - e)))
                    E[p, h, o // BLOCK] = e
                    y = new * 2.0 ** -e
                    X[p, h, o + lo - b * BLOCK:o + hi - b * BLOCK] = torch.where(torch.isfinite(y), e4m3(y), math.nan)


def attend(cache, q, table, q_start, kv_len, causal):
    """[tokens, Hq, d] fp64, and a bound on the error of the kernel's result.

    The bound: o is rounded to bf16 (2^-8 of it) and p before the product with V (2^-8 of each p, so of
    sum p |v|).  A score's error moves its p by that much, relatively: Q is held to 2^-22 of its row's
    largest magnitude m (so m sum |k| 2^-22), the products are summed in fp32 (128 terms, at most 2^-20 of
    sum |q k| in the order of the matrix core and over four products), and its product with the scale, the
    subtraction of the maximum and exp2 add 2^-21 of |s| + |max|; l and O~ gain at most 2^-18 in a chain of up
    to 2^12 fp32 additions whose errors are random."""
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    Hq, Hkv = q.shape[1], cache.k.shape[1]
    for s in range(len(kv_len)):
        n, L = q_start[s + 1] - q_start[s], kv_len[s]
        for h in range(Hkv if n else 0):
            k, v = cache.rows(table[s], L, h)
            for g in range(Hq // Hkv):
                i = h * (Hq // Hkv) + g
                x = q[q_start[s]:q_start[s + 1], i].double()
                t = x @ k.t() / math.sqrt(D)
                end = torch.arange(L - n + 1, L + 1) if causal else torch.full((n,), L)
                hidden = torch.arange(L) >= end[:, None]
                err = (2.0 ** -22 * x.abs().amax(-1, keepdim=True) * k.abs().sum(-1)
                       + 2.0 ** -20 * x.abs() @ k.abs().t()) / math.sqrt(D)
                t = t.masked_fill(hidden, -math.inf)
                m = t.amax(-1, keepdim=True) if L else torch.zeros(n, 1)
                m = torch.where(m == -math.inf, 0.0, m)
                p = torch.exp(t - m)
                l = p.sum(-1, keepdim=True)
                some = (l > 0) | l.isnan()
                p = torch.where(some, p / l, 0.0)
                # 0 * NaN: a hidden key's value does not count
                vv = torch.where(torch.isnan(v), 0.0, v)
                nan = ((~hidden).double() @ torch.isnan(v).double() > 0) if L else torch.zeros(n, D, dtype=bool)
                o = torch.where(nan, math.nan, p @ vv)
                rel = 2 * err + 2.0 ** -21 * (torch.where(hidden, 0.0, t.abs()) + m.abs())
                rel = torch.where(hidden, 0.0, rel)
                drift = rel.amax(-1, keepdim=True) if L else torch.zeros(n, 1)
                out[q_start[s]:q_start[s + 1], i] = o
                tol[q_start[s]:q_start[s + 1], i] = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -17 + 2 * drift) * (p @ vv.abs())
    return out, tol
