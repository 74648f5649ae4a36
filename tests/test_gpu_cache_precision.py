"""What attention over the cache keeps of its probabilities and values.

Tolerance: cache_reference.attend's bound with p's rounding to f16 in the place of 2^-8: half a step, 2^-11 of each p,
so 2^-11 of sum p |v|.  (p below 2^-25 of the largest is rounded by 2^-36 of that: no p is so small where the values
differ much.)  The rest of that bound (the result's own rounding 2^-8 |o|, the scores' errors, sums in fp32) stays."""
import pytest

import cache_reference as ref
from test_gpu_cache import batch, empty_cache, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# bounds that choose one workgroup per item, shares by wave and tiles of 128 rows
WAYS = {"items": (12, 200), "shares": (1, 5000), "tiles": (100, 5000)}


def check(got, cache, q, table, start, lens, causal):
    """`got` against 64 bits: the bound with 2^-11 for 2^-8 of sum p |v|."""
    c = ref.Cache(*cache)
    want, loose = ref.attend(c, q.cpu(), table, start, lens, causal)
    c.v = c.v.abs()
    size, _ = ref.attend(c, q.cpu(), table, start, lens, causal)  # sum p |v|
    err = (got.cpu().double() - want).abs()
    tol = loose - (2.0 ** -8 - 2.0 ** -11) * size
    assert bool((err <= tol + 1e-38).all()), float((err / (tol + 1e-38)).max())


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("keys", [2, 3, 7, 31, 100])
def test_probabilities_hold_11_bits(mx, keys, way):  # noqa: F811
    """Few keys, whose rounding errors do not average out, over values that nearly cancel in many channels."""
    print(f"[precision] {keys} {way}", flush=True)
    table, start, lens, pages = batch([2] * 20, [keys - 2] * 20, 32, seed=keys)
    cache = filled(mx, pages, 2, 32, keys)
    q = rows(start[-1], 8, 5, 0.2)
    got = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), False, *WAYS[way])
    check(got, cache, q, table, start, lens, False)


SPREADS = {
    "up": [-50, -30, -20, -10, 0, 7, 8, 30],
    "down": [30, 14, 13, 0, -1, -10, -20, -24],
    "both": [0, 20, -20, 23, -25, 7, -15, 8],
    "smallest": [-130, -125, -120, -110, -100, -112, -128, -133],
    "largest": [100, 110, 120, 126, 127, 110, 105, 127],
}


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("spread", list(SPREADS))
@pytest.mark.parametrize("causal", [True, False])
def test_values_of_very_different_blocks(mx, causal, spread, way):  # noqa: F811
    """Blocks of 32 values around powers of two up to 2^54 apart; a query for every block that it is the last to see,
    so that rows of one tile hold sums of very different magnitudes."""
    print(f"[precision] {spread} {way} {causal}", flush=True)
    powers = SPREADS[spread]
    n = 32 * len(powers)
    g = torch.Generator().manual_seed(2)
    k, v = rows(n, 1, 3, 0.3), torch.randn((n, 1, ref.D), generator=g).clamp(-1.7, 1.7)
    v = (v.view(-1, 32, 1, ref.D).double() * torch.tensor([2.0 ** p for p in powers], dtype=torch.float64).view(-1, 1, 1, 1))
    v = v.view(n, 1, ref.D).to(torch.bfloat16).cuda()
    cache = empty_cache(mx, n // 32, 1, 32)
    table = torch.arange(n // 32, dtype=torch.int32)[None]
    mx.cache_append(k, v, *cache, table.cuda(), ints([0, n]), ints([n]))
    q = rows(n, 2, 4, 0.3)
    got = mx.cache_attend(q, *cache, table.cuda(), ints([0, n]), ints([n]), causal, *WAYS[way])
    check(got, cache, q, table, [0, n], [n], causal)


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("power", [10, 18, 20, 22, 23, 24])
def test_scores_of_large_magnitude(mx, power, way):  # noqa: F811
    """Sums q.k of up to 3 * 2^(power + 4): the largest takes everything, whatever the rounding of its own product with
    the scale does to p, so the result is its key's value, rounded to f16's product and bf16.  (The scores that the
    call takes, q.k / sqrt(128), end at 2^26.)"""
    print(f"[precision] scores 2^{power} {way}", flush=True)
    n = 64
    k = torch.zeros((n, 1, ref.D))
    k[:, 0, 0] = torch.tensor([float((5 * i) % 8 + 1) for i in range(n)])  # 1 to 8 eighths, eight keys of each
    k[:, 0, 1] = torch.tensor([1.0 if i == 37 else 0.0 for i in range(n)])
    v = torch.randn((n, 1, ref.D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    cache = empty_cache(mx, 2, 1, 32)
    table = torch.tensor([[0, 1]], dtype=torch.int32)
    mx.cache_append(k.to(torch.bfloat16).cuda(), v, *cache, table.cuda(), ints([0, n]), ints([n]))
    q = torch.zeros((6, 2, ref.D))
    q[:, 0, 0], q[:, 0, 1] = 2.0 ** power, 2.0 ** (power + 4)      # key 37 by far
    q[:, 1, 0], q[:, 1, 1] = -2.0 ** power, 2.0 ** (power + 4) * 3  # and from below
    got = mx.cache_attend(q.to(torch.bfloat16).cuda(), *cache, table.cuda(), ints([0, 6]), ints([n]), False, *WAYS[way])
    want = ref.Cache(*cache).rows(table[0], n, 0)[1][37]
    assert bool(((got.cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -11) * want.abs()).all())


@pytest.mark.parametrize("way", list(WAYS))
def test_a_scale_that_is_no_number_reaches_every_row_that_sees_it(mx, way):  # noqa: F811
    cache = filled(mx, 4, 1, 32, 3)
    table = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32).cuda()
    cache[3][1] = 255
    got = mx.cache_attend(rows(6, 2, 4), *cache, table, ints([0, 6]), ints([128]), False, *WAYS[way])
    assert bool(got.isnan().all())
