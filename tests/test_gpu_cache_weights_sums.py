"""Weights of keys where scores are large: every kernel that makes them divides by the sum of the scores that it weighs,
so a row's probabilities add up to 1 whatever the scores' size and whichever way the caller's bounds choose."""
import math

import pytest

import cache_reference as ref
import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

WIDE = 1 << 24  # keys of a table so wide that scores are not kept

# new, past, Hq, Hkv, page, max_q, max_kv
WAYS = [
    ([1, 3], [900, 500], 8, 2, 64, 3, 1000),       # few short keys, scores kept
    ([40, 60], [300, 900], 8, 2, 64, 60, 1000),    # few short keys, computed again
    ([1, 3], [2900, 500], 8, 2, 64, 3, 3000),      # long ones, scores kept
    ([1, 3], [2900, 500], 32, 2, 4096, 1, WIDE),   # long ones, computed again
    ([40, 150], [2900, 1300], 8, 2, 64, 150, 3000),  # tiles of 128 rows, computed again
    ([40, 150], [2900, 1300], 6, 2, 64, 150, 3000),  # (of heads that no step of rows divides)
    ([1500], [10], 4, 4, 128, 1500, 1600),         # prompts
]


@pytest.mark.parametrize("scale", [1.0, 40.0])
@pytest.mark.parametrize("way", WAYS)
def test_rows_add_up_to_one(mx, way, scale):  # noqa: F811
    """The sum over a sequence's keys is the number of its rows.  l is a sum of the same p in chains of at most 16 + 94
    additions (3000 keys) that lose 2^-24 each; moved from one running maximum to another and cut by rounding of s c - m, a p
    above 2^-25 loses at most 25 2^-24 and four roundings more, 1 / l and its product two; the weights add a row's p in
    chains of at most 1500 terms of which half an ulp each is lost, random in sign: 2^-24 of the sum in the worst case
    each, sqrt(1500) of those as they fall.  In all below 2^-24 (110 + 29 + 2 + 39) < 2^-16 of the rows."""
    new, past, Hq, Hkv, page, max_q, max_kv = way
    print(f"[sums] {way} {scale}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    if max_kv == WIDE:
        table = torch.cat((table, torch.full((len(new), WIDE // page - table.shape[1]), 1 << 30, dtype=torch.int32)), 1)
    q = rows(start[-1], Hq, 5, scale)
    w = mx.cache_attend_weights(q, *cache, table.cuda(), ints(start), ints(lens), None, True, max_q, max_kv)[1].cpu()
    for s, n in enumerate(new):
        for h in range(Hkv):
            got = steps.weights_of(w, table[s], lens[s], h).double()
            want = n * Hq // Hkv
            assert bool((got >= 0).all())
            assert abs(float(got.sum()) - want) <= 2.0 ** -16 * want, (s, h, float(got.sum()), want)


def test_no_way_gives_other_weights(mx):  # noqa: F811
    """The same batch by every kernel, rows of large scores: as the same numbers are summed over, the weights agree
    within the roundings named above, 2^-16 of themselves and, of each row's p, 2^-24 of the distance of scores (p above
    2^-25; smaller ones by 2^-40)."""
    new, past, page = [3, 1], [900, 500], 64
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, 2, page, 7)
    q = rows(start[-1], 8, 5, 40.0)
    args = (q, *cache)
    wide = torch.cat((table, torch.full((2, WIDE // page - table.shape[1]), 1 << 30, dtype=torch.int32)), 1)
    got = []
    for t, bounds in ((table, (3, 903)), (table, (40, 960)), (table, (1, 0)), (wide, (1, 2000)), (wide, (1, 0)), (wide, (40, 2000))):
        w = mx.cache_attend_weights(*args, t.cuda(), ints(start), ints(lens), None, True, *bounds)[1].cpu()
        got.append(torch.cat([steps.weights_of(w, table[s], lens[s], h) for s in range(2) for h in range(2)]).double())
    assert math.isfinite(float(got[0].sum()))
    for x in got[1:]:
        assert bool(((x - got[0]).abs() <= 2.0 ** -16 * got[0] + 2.0 ** -40).all())
