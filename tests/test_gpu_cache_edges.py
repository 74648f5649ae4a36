"""Calls at the edges of what the paged cache's operators take; bounds as in test_gpu_cache.py."""
import math

import pytest

import cache_reference as ref
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

GUARD = 4096


def guarded_cache(mx, pages, heads, page):  # noqa: F811
    """A cache of zeros whose arrays lie between bytes of 7, and what holds them."""
    shapes = mx.cache_shapes(pages, heads, page)
    room = [torch.full((math.prod(s) + 2 * GUARD,), 7, dtype=torch.uint8, device="cuda") for s in shapes]
    cache = [x[GUARD:-GUARD].view(s).zero_() for x, s in zip(room, shapes)]
    return cache, room


def untouched(room, out, tokens):
    """The bytes around the cache, and the rows of 9 around the call's."""
    torch.cuda.synchronize()
    return (all(bool((x[:GUARD] == 7).all() and (x[-GUARD:] == 7).all()) for x in room)
            and bool((out[:-tokens - 64] == 9).all() and (out[-64:] == 9).all()))


@pytest.mark.parametrize("start", [[0, 90, 50], [-7, -3, 1 << 30], [50, 20, 0], [5, 5, 5]])
def test_starts_of_no_batch_write_nothing_around(mx, start):  # noqa: F811
    print(f"[starts] {start}", flush=True)
    cache, room = guarded_cache(mx, 4, 1, 32)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).cuda()
    k = rows(50, 1, 1)
    out = torch.full((64 + 50 + 64, 1, ref.D), 9.0, dtype=torch.bfloat16, device="cuda")
    mx.cache_append(k, k, *cache, table, ints(start), ints([64, 64]))
    mx.cache_attend(k, *cache, table, ints(start), ints([64, 64]), out=out[64:-64])
    assert untouched(room, out, 50)


@pytest.mark.parametrize("max_q", [1, 0])
def test_starts_whose_work_passes_32_bits(mx, max_q):  # noqa: F811
    """1024 sequences that each claim all of the call's 8192 tokens: 2^18 rows and 2^10 blocks of keys each, 2^33
    units in all, for which a call of these sizes has 2^24 at most."""
    tokens, seqs, group = 8192, 2048, 32
    print(f"[starts] passing 32 bits, max_q {max_q}", flush=True)
    cache, room = guarded_cache(mx, 8, 1, 4096)
    table = torch.arange(8, dtype=torch.int32, device="cuda").expand(seqs, 8).contiguous()
    g = torch.Generator().manual_seed(1)
    lens = torch.tensor([64, 20000, 32768], dtype=torch.int32)[torch.randint(3, (seqs,), generator=g)].cuda()
    q = rows(tokens, group, 1)
    out = torch.full((64 + tokens + 64, group, ref.D), 9.0, dtype=torch.bfloat16, device="cuda")
    mx.cache_attend(q, *cache, table, ints([0, tokens] * (seqs // 2) + [0]), lens, max_q=max_q, out=out[64:-64])
    assert untouched(room, out, tokens)
    # the same sizes with an ascending start: one token for each of the first sequences
    st = torch.arange(seqs + 1, dtype=torch.int32, device="cuda")
    a = mx.cache_attend(q, *cache, table, st, lens, max_q=max_q)
    assert bool((a[:seqs] == 0).all())  # values of zero


# bounds that choose one workgroup per item, shares by wave and tiles of 128 rows
WAYS = {"items": (12, 200), "shares": (1, 5000), "tiles": (100, 5000)}


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("what", ["page", "value scale", "key scale"])
def test_last_block_without_numbers_reaches_only_the_rows_that_see_it(mx, what, way):  # noqa: F811
    """A page that is not there while page 0, which stands in for it, holds no numbers, and a block whose scale byte
    is E8M0's NaN: NaN for the tokens that see that block, and no other bits for those before it."""
    print(f"[edges] {what} {way}", flush=True)
    cache = filled(mx, 6, 2, 32, 3)
    for c in cache:
        c[0] = 0xFF
    kc, ks, vc, vs = cache
    q = rows(12, 4, 4)
    table = torch.tensor([[3, 4, 5]], dtype=torch.int32)
    args = ints([0, 12]), ints([70]), True, *WAYS[way]  # positions 58 to 69: the last block from token 6 on
    clean = mx.cache_attend(q, *cache, table.cuda(), *args)
    assert bool(clean.isfinite().all())
    if what == "page":
        table[0, 2] = 99
    elif what == "value scale":
        vs[5] = 255
    else:
        ks[5] = 255
    got = mx.cache_attend(q, *cache, table.cuda(), *args)
    assert torch.equal(got[:6], clean[:6])
    assert bool(got[6:].isnan().all())


@pytest.mark.parametrize("way", list(WAYS))
def test_queries_that_see_nothing_get_zero_whatever_they_hold(mx, way):  # noqa: F811
    """More new tokens than the sequence has keys: those before the first key are zero, infinite and NaN queries
    among them, beside rows of the same tile that see keys."""
    print(f"[edges] unseen {way}", flush=True)
    cache = filled(mx, 3, 2, 32, 3)
    table = torch.tensor([[1, 2]], dtype=torch.int32).cuda()
    q = rows(12, 4, 4)
    args = table, ints([0, 12]), ints([7]), True, *WAYS[way]  # tokens 0 to 4 are before position 0
    clean = mx.cache_attend(q, *cache, *args)
    q[0, 0, 3], q[1, 1, 100], q[2], q[4, 3, 0] = math.inf, math.nan, -math.inf, math.nan
    q[6, 2, 5] = math.inf  # this one sees keys
    got = mx.cache_attend(q, *cache, *args)
    assert bool((got[:5] == 0).all())
    assert bool(got[6, 2].isnan().all())
    clean[6, 2] = got[6, 2] = 0
    assert torch.equal(got, clean)
