"""Attention over the paged cache where scores are large, within what the header states of them: sums of the FP8 matrix
cores, off by up to 2^-15 of sum |q k|, of queries held to 2^-21 of their row's largest magnitude.  (Beside small scores
these are below the rounding of the output.)"""
import math

import pytest

import cache_reference as ref
import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401
from test_gpu_cache_window import parents_mask, random_parents

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def expected(cache, q, table, start, lens, sees, fp8):
    """Output in 64 bits and the bound of its error: bf16 of it and of each p (f16: less) 2^-8, 2^-17 for l and O's sums, and
    what the scores' errors move p and l by: each twice that of a score (its maximum's and its own), exp2's 2^-21
    of it and of the maximum, exp(x) - 1 < 1.2 x below 0.3."""
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    group = q.shape[1] // cache.k.shape[1]
    for s, L in enumerate(lens):
        tokens = slice(start[s], start[s + 1])
        hidden = ~sees(start[s + 1] - start[s], L, tokens)
        for i in range(q.shape[1]):
            k, v = cache.rows(table[s], L, i // group)
            x = q[tokens, i].double()
            t = (x @ k.t() / math.sqrt(ref.D)).masked_fill(hidden, -math.inf)
            m = t.amax(-1, keepdim=True)
            p = torch.softmax(t, -1)
            size = x.abs() @ k.abs().t()
            err = (2.0 ** -15 * size + 2.0 ** -21 * x.abs().amax(-1, keepdim=True) * k.abs().sum(-1) if fp8
                   else 2.0 ** -20 * size) / math.sqrt(ref.D)
            rel = torch.where(hidden, 0.0, 2 * err + 2.0 ** -21 * (t.abs().masked_fill(hidden, 0.0) + m.abs()))
            near = torch.where(p > 0, rel, 0.0).amax(-1, keepdim=True)
            assert float(near.max()) < 0.3
            out[tokens, i] = p @ v
            tol[tokens, i] = 2.0 ** -8 * (p @ v).abs() + (2.0 ** -8 + 2.0 ** -17 + 2.4 * near) * (p @ v.abs())
    return out, tol


@pytest.mark.parametrize("scale", [4.0, 20.0])
@pytest.mark.parametrize("bounds", [(0, 0), (1, 1000), (1, 5000), (64, 5000)])
def test_outputs_of_large_scores(mx, bounds, scale):  # noqa: F811
    new, past, page = [1, 40, 6], [900, 300, 700], 64
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, 2, page, 7)
    n = start[-1]
    # rows of one size: no row's scores so large that the bound says nothing
    q = (rows(n, 8, 5).float() / rows(n, 8, 5).float().norm(dim=-1, keepdim=True) * math.sqrt(ref.D) * scale).to(torch.bfloat16)
    mask = torch.cat([parents_mask(random_parents(a, s), 2) for s, a in enumerate(new)])
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    values = ref.Cache(*cache)
    weights = lambda: mx.cache_attend_weights(*args, None, True, *bounds)[0]  # noqa: E731
    for got, sees, fp8 in ((lambda: mx.cache_attend(*args, True, *bounds), steps.causal, True),
                           (lambda: mx.cache_attend_window(*args, 200, 9, True, *bounds), steps.window(200, 9, True), True),
                           (lambda: mx.cache_attend_tree(*args, mask.cuda(), *bounds), steps.tree(mask), True),
                           (weights, steps.causal, False)):
        want, tol = expected(values, q.cpu(), table, start, lens, sees, fp8)
        if got is weights and 0 < bounds[1] < max(lens):
            continue
        err = (got().cpu().double() - want).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
