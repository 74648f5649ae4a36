"""Attention over the paged cache with a sliding window and sinks, and for trees of drafted tokens, against 64 bits
(the bound of cache_reference.attend)."""
import pytest

import cache_reference as ref
import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

WINDOWS = [
    # new, past, Hq, Hkv, page, causal, window, sinks
    ([1], [0], 1, 1, 32, True, 1, 0),
    ([1], [31], 2, 2, 32, True, 1, 1),
    ([1, 1, 1], [32, 0, 63], 8, 1, 32, True, 32, 0),
    ([1, 1], [2500, 4099], 24, 24, 256, False, 1000, 4),
    ([1] * 40, [97 * i % 701 for i in range(40)], 32, 8, 32, True, 100, 5),
    # more than one share, in and out of the window
    ([1, 1, 1], [9000, 20000, 50], 8, 2, 64, True, 4096, 4),
    ([4, 3], [6000, 1], 10, 2, 128, True, 2000, 33),
    ([1], [40000], 1, 1, 256, False, 30001, 31),
    # sinks that reach into the window, that are longer than it, and than the sequence
    ([33], [0], 3, 3, 32, True, 8, 16),
    ([70], [200], 4, 2, 64, True, 64, 100),
    ([5, 0, 70], [0, 50, 31], 4, 2, 64, True, 40, 1000),
    ([100], [300], 5, 1, 256, False, 33, 32),
    # tiles of 128 rows: windows that begin inside a block, prompts many windows long
    ([257], [1000], 2, 2, 128, True, 127, 3),
    ([300, 3, 129], [5, 4000, 64], 8, 2, 64, True, 1500, 64),
    ([700], [0], 4, 1, 32, True, 1100, 0),
    ([1500], [3000], 1, 1, 64, True, 1025, 7),
    ([40], [20000], 4, 1, 256, True, 5000, 40),
    ([200], [7000], 3, 3, 128, False, 2000, 700),
    # many sequences, some without tokens, some without keys
    ([i % 3 for i in range(300)], [(37 * i) % 90 for i in range(300)], 4, 2, 32, True, 17, 2),
    ([2], [70], 256, 1, 32, True, 20, 0),
]


def check(o, want, tol, n):
    err = (o.cpu().double() - want)[:n].abs()
    assert bool((err <= tol[:n] + 1e-30).all()), float((err / (tol[:n] + 1e-30)).max())


@pytest.mark.parametrize("case", WINDOWS)
def test_window_against_64_bits(mx, case):  # noqa: F811
    new, past, Hq, Hkv, page, causal, size, sinks = case
    print(f"[window] {str(case)[:120]}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    T = start[-1] + 2
    q = rows(T, Hq, 5, 0.5)
    out = torch.full((T, Hq, ref.D), 3.0, dtype=torch.bfloat16, device="cuda")
    args = (q, *cache, table.cuda(), ints(start), ints(lens), size, sinks, causal)
    mx.cache_attend_window(*args, out=out)
    want, tol, _ = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.window(size, sinks, causal))
    n = start[-1]
    check(out, want, tol, n)
    assert bool((out[n:] == 3).all())  # tokens of no sequence are left alone
    for bounds in ((max(new), max(lens)), (1, 1), (1, 5000), (33, 5000)):  # which kernel
        check(mx.cache_attend_window(*args, *bounds), want, tol, n)


def test_a_window_over_all_keys_is_plain_attention(mx):  # noqa: F811
    """Also the largest numbers that the call takes."""
    table, start, lens, pages = batch([1, 50, 300], [5000, 70, 900], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(start[-1], 8, 5)
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    for causal in (True, False):
        want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, causal)
        for w, a in ((1 << 40, 0), (1, 1 << 40), (6000, 7000)):
            check(mx.cache_attend_window(*args, w, a, causal), want, tol, start[-1])


def test_pages_that_no_token_sees_are_not_read(mx):  # noqa: F811
    """Table entries between sinks and window may be anything."""
    for new, past in (([1], [3000]), ([50], [3000]), ([8], [700])):
        table, start, lens, pages = batch(new, past, 32)
        cache = filled(mx, pages, 2, 32, 3)
        q = rows(start[-1], 6, 4)
        gone = table.clone()
        gone[0, 3:(past[0] + 1 - 100) // 32] = -1  # sinks: 90 tokens, pages 0 .. 2
        a, b = (mx.cache_attend_window(q, *cache, t.cuda(), ints(start), ints(lens), 100, 90) for t in (table, gone))
        assert torch.equal(a, b) and bool(a.isfinite().all())
        gone[0, 1] = pages  # a sink's
        c = mx.cache_attend_window(q, *cache, gone.cuda(), ints(start), ints(lens), 100, 90)
        assert bool(c.isnan().all())


@pytest.mark.parametrize("new", [1, 6, 70])
def test_masked_nan_does_not_reach_a_window(mx, new):  # noqa: F811
    """NaN codes and scales in keys before the window, in its first block and between the sinks and it."""
    page, past, size, sinks = 64, 500, 77, 10
    table, start, lens, pages = batch([new], [past], page, spare=1)
    cache = filled(mx, pages, 2, page, 3)
    q = rows(new, 6, 4)
    args = (table.cuda(), ints(start), ints(lens), size, sinks)
    clean = mx.cache_attend_window(q, *cache, *args)
    kc, ks, vc, vs = (c.clone() for c in cache)
    K, V = kc.view(pages, 2, page // 32, 8, 32, 16).transpose(3, 4), vc.transpose(3, 4)
    first = past + 1 - size  # of the first token's window
    for t in range(sinks, first):
        p, o = int(table[0, t // page]), t % page
        K[p, :, o // 32, o % 32] = 0x7F
        V[p, :, o // 32, o % 32] = 0x7F
    for t in range(32, first - first % 32, 32):  # whole blocks
        ks[int(table[0, t // page]), :, t % page // 32] = 255
        vs[int(table[0, t // page]), :, t % page // 32] = 255
    got = mx.cache_attend_window(q, kc, ks, vc, vs, *args)
    assert torch.equal(clean, got)


def test_window_repeats_bit_for_bit_and_in_a_graph(mx):  # noqa: F811
    table, start, lens, pages = batch([1, 1, 40], [3000, 10, 5000], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(42, 8, 5)
    args = (q, *cache, table.cuda(), ints(start), ints(lens), 2000, 9)
    a = mx.cache_attend_window(*args)
    assert torch.equal(a, mx.cache_attend_window(*args))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b = mx.cache_attend_window(*args)
    for _ in range(3):
        b.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        mx.cache_attend_window(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c = mx.cache_attend_window(*args, stream=s)
    s.synchronize()
    assert torch.equal(a, c)


# ---------------------------------------------------------------------------


def parents_mask(parents, words):
    """Masks of trees given by each token's parent among the drafts (-1: none)."""
    out, seen = [], []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        out.append([seen[i] >> 32 * w & 0xFFFFFFFF for w in range(words)])
    t = torch.tensor(out, dtype=torch.int64).view(len(parents), words)
    return torch.where(t >= 1 << 31, t - (1 << 32), t).to(torch.int32)


def random_parents(n, seed):
    g = torch.Generator().manual_seed(seed)
    return [int(torch.randint(-1, i, (1,), generator=g)) if i else -1 for i in range(n)]


TREES = [
    # new, past, Hq, Hkv, page, words
    ([1], [0], 1, 1, 32, 1),
    ([7], [500], 8, 8, 32, 1),
    ([2, 5, 7], [10, 127, 31], 10, 2, 128, 1),
    ([32], [32], 1, 1, 32, 1),
    ([33, 1, 31], [31, 5, 33], 2, 1, 64, 2),
    ([64, 60, 0, 3], [1, 2000, 10, 5000], 8, 2, 64, 2),
    ([25] * 5, [1500, 6000, 0, 77, 900], 40, 8, 128, 1),
    ([200], [45], 2, 2, 32, 7),
    ([8], [3000], 16, 4, 64, 1),
    ([4, 2], [9000, 2100], 8, 2, 64, 3),
    ([i % 4 for i in range(270)], [(37 * i) % 90 for i in range(270)], 4, 2, 32, 1),
]


@pytest.mark.parametrize("case", TREES)
def test_tree_against_64_bits(mx, case):  # noqa: F811
    new, past, Hq, Hkv, page, words = case
    print(f"[tree] {str(case)[:120]}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    T = start[-1] + 2
    mask = torch.cat([parents_mask(random_parents(n, s), words) for s, n in enumerate(new)] + [torch.full((2, words), -1)])
    mask = mask.to(torch.int32)
    q = rows(T, Hq, 5, 0.5)
    out = torch.full((T, Hq, ref.D), 3.0, dtype=torch.bfloat16, device="cuda")
    args = (q, *cache, table.cuda(), ints(start), ints(lens), mask.cuda())
    mx.cache_attend_tree(*args, out=out)
    want, tol, _ = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.tree(mask))
    n = start[-1]
    check(out, want, tol, n)
    assert bool((out[n:] == 3).all())
    for bounds in ((max(new), max(lens)), (1, 1), (1, 5000), (33, 5000)):
        check(mx.cache_attend_tree(*args, *bounds), want, tol, n)


@pytest.mark.parametrize("bounds", [(1, 1), (1, 5000), (64, 5000)])
def test_tree_masks_of_any_bits(mx, bounds):  # noqa: F811
    """Bits of no token, of later ones, none at all, words that end before the drafts, and drafts without a past:
    some rows see nothing and get 0, whatever they hold."""
    new, past = [40, 9, 33], [0, 3, 0]
    table, start, lens, pages = batch(new, past, 32)
    cache = filled(mx, pages, 2, 32, 7)
    g = torch.Generator().manual_seed(1)
    mask = torch.randint(-1 << 31, 1 << 31, (82, 1), generator=g).to(torch.int32)
    mask[5] = 0
    mask[60] = 0
    q = rows(82, 4, 5)
    q[5] = float("nan")
    args = (q, *cache, table.cuda(), ints(start), ints(lens), mask.cuda())
    o = mx.cache_attend_tree(*args, *bounds)
    want, tol, _ = steps.attend(ref.Cache(*cache), torch.nan_to_num(q.cpu()), table, start, lens, steps.tree(mask))
    check(o, want, tol, 82)
    assert bool((o[5] == 0).all()) and bool((o[60] == 0).all())


def test_a_chain_is_causal_attention(mx):  # noqa: F811
    """More new tokens than keys too: the first ones see nothing."""
    for new, past, lens in (([6, 40], [1000, 0], None), ([8], [0], [5])):
        table, start, L, pages = batch(new, past, 64)
        lens = lens or L
        cache = filled(mx, pages, 2, 64, 7)
        q = rows(start[-1], 8, 5)
        mask = torch.cat([parents_mask(list(range(-1, n - 1)), 2) for n in new]).cuda()
        if lens is not L:  # (tokens without a place: no bit names them)
            mask &= torch.tensor([~0b111, -1], dtype=torch.int32, device="cuda")
        o = mx.cache_attend_tree(q, *cache, table.cuda(), ints(start), ints(lens), mask)
        want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, True)
        check(o, want, tol, start[-1])


def test_tree_in_a_graph_with_new_masks(mx):  # noqa: F811
    table, start, lens, pages = batch([20, 12], [2000, 300], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(32, 8, 5)
    masks = [torch.cat([parents_mask(random_parents(n, s + i), 1) for s, n in enumerate((20, 12))]).cuda() for i in (0, 7)]
    now = masks[0].clone()
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    mx.cache_attend_tree(*args, now)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b = mx.cache_attend_tree(*args, now)
    for m in masks + masks:
        now.copy_(m)
        g.replay()
        assert torch.equal(b, mx.cache_attend_tree(*args, m))
