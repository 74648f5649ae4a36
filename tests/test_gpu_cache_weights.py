"""Attention that weighs the cache's keys, against 64 bits (bounds of cache_steps_reference.attend)."""
import math

import pytest

import cache_reference as ref
import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

WEIGHTS = [
    # new, past, Hq, Hkv, page, causal
    ([1], [0], 1, 1, 32, True),
    ([1, 1, 1], [32, 0, 63], 8, 1, 32, True),
    ([1], [500], 40, 8, 64, False),
    ([2, 1, 3, 4], [10, 127, 128, 1000], 10, 2, 128, True),
    ([33], [0], 3, 3, 32, True),
    ([5, 0, 70], [0, 50, 31], 4, 2, 64, True),
    ([100], [300], 5, 1, 256, False),
    ([1, 1, 1], [9000, 20000, 50], 8, 2, 64, True),
    ([1, 1], [2500, 4099], 24, 24, 256, False),
    ([257, 60], [1000, 2000], 2, 2, 128, True),
    ([300, 3], [5, 4000], 8, 8, 64, False),
    ([700], [0], 4, 1, 32, True),
    ([i % 3 for i in range(300)], [(37 * i) % 90 for i in range(300)], 4, 2, 32, True),
    ([2], [70], 256, 1, 32, True),
    ([40], [5000], 4, 1, 256, True),
]


def check(w, want, before, table, start, lens, near=False):
    """Weights w of every sequence with tokens against the sums `want` and what was there before; near: few rows."""
    used = torch.zeros(w.shape, dtype=torch.bool)
    for (s, h), (total, *bounds) in want.items():
        bound = bounds[near]
        L, n = lens[s], start[s + 1] - start[s]
        old = steps.weights_of(before, table[s], L, h).double() if before is not None else torch.zeros(L, dtype=torch.float64)
        old[max(L - n, 0):] = 0
        got = steps.weights_of(w, table[s], L, h).double()
        sum_ = old + total
        tol = bound + 2.0 ** -23 * sum_.abs() + 1e-30
        bad = (got - sum_).abs() > tol
        assert not bool(bad.any()), (s, h, int(bad.nonzero()[0]), float(((got - sum_).abs() / tol).max()))
        t = torch.arange(L)
        used[table[s][t // w.shape[2]].long(), h, t % w.shape[2]] = True
    return used


@pytest.mark.parametrize("case", WEIGHTS)
def test_weights_against_64_bits(mx, case):  # noqa: F811
    new, past, Hq, Hkv, page, causal = case
    print(f"[weights] {str(case)[:120]}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    T = start[-1] + 2
    q = rows(T, Hq, 5, 0.5)
    before = torch.rand((pages, Hkv, page), generator=torch.Generator().manual_seed(3)) * 3
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    want, tol, sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens,
                                   steps.causal if causal else steps.everything)
    n = start[-1]
    for bounds in ((0, 0), (max(new), max(lens)), (1, max(lens)), (33, max(lens)), (1, 6000), (129, 30000)):
        if bounds[1] and bounds[1] < max(lens):
            continue
        near = bounds[1] > 0 and min(bounds[0], start[-1] + 2) * Hq // Hkv <= 32 and max(new) * Hq // Hkv <= 64
        o, w = mx.cache_attend_weights(*args, before.cuda(), causal, *bounds,
                                       weights_out=torch.full_like(before, -7.0, device="cuda"))
        err = (o.cpu().double() - want)[:n].abs()
        assert bool((err <= tol[:n] + 1e-30).all())
        used = check(w.cpu(), sums, before, table, start, lens, near)
        assert bool((w.cpu()[~used] == -7).all())  # nothing else is written
    # in place and from nothing
    o, w = mx.cache_attend_weights(*args, None, causal)
    check(w.cpu(), sums, None, table, start, lens)
    w = before.cuda()
    assert mx.cache_attend_weights(*args, w, causal)[1] is w
    used = check(w.cpu(), sums, before, table, start, lens)
    assert torch.equal(w.cpu()[~used], before[~used])


def test_every_row_gives_one_and_repeats(mx):  # noqa: F811
    """Every row's probabilities sum to 1 (4 heads a group and the new tokens), and equal calls give equal bits."""
    table, start, lens, pages = batch([1, 1, 40], [3000, 10, 5000], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(42, 8, 5)
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.causal)[2]
    for bounds in ((1, 6000), (40, 6000)):
        o, w = mx.cache_attend_weights(*args, None, True, *bounds)
        for s, n in enumerate((1, 1, 40)):
            for h in range(2):
                total = float(steps.weights_of(w.cpu(), table[s], lens[s], h).double().sum())
                assert abs(total - 4 * n) <= float(sums[s, h][1].sum())
        o2, w2 = mx.cache_attend_weights(*args, None, True, *bounds)
        assert torch.equal(w, w2) and torch.equal(o, o2)


def test_scores_too_many_to_keep(mx):  # noqa: F811
    """More than 1 GiB of scores are not kept but computed again: the same weights, of one long table and of many short
    sequences."""
    table, start, lens, pages = batch([1], [900], 4096)
    cache = filled(mx, pages, 2, 4096, 7)
    q = rows(1, 64, 5)
    wide = torch.cat((table, torch.full((1, 4094), 1 << 30, dtype=torch.int32)), 1).cuda()
    sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.causal)[2]
    for max_kv in (901, 0):  # 0: up to 2^24 keys, 4 GiB of scores
        w = mx.cache_attend_weights(q, *cache, wide, ints(start), ints(lens), None, True, 1, max_kv)[1]
        check(w.cpu(), sums, None, table, start, lens)
    S = 20000
    t = torch.arange(S, dtype=torch.int32).view(S, 1)
    cache = filled(mx, S, 1, 32, 3)
    lens = [1 + 7 * i % 32 for i in range(S)]
    q = rows(S, 16, 6)
    args = (q, *cache, t.cuda(), ints(list(range(S + 1))), ints(lens))
    (a, v), (b, w) = (mx.cache_attend_weights(*args, None, True, 1, m) for m in (32, 0))
    t32 = torch.cat((t, torch.full((S, 31), -1, dtype=torch.int32)), 1).cuda()
    c, x = mx.cache_attend_weights(q, *cache, t32, *args[-2:], None, True, 1, 1024)
    assert torch.equal(v, w)  # (a table of 32 keys)
    # the same scores, but l of the FP8 ones: 2^-15 of sum |q k| and two roundings in 2^-20
    k = ref.Cache(*cache)
    size = float(q.float().norm(dim=-1).max()) * float((k.k * torch.exp2(k.ke.double())[..., None, None].amax()).norm(dim=-1).max())
    rel = 2.0 ** -15 * size / math.sqrt(ref.D) + 2.0 ** -18
    assert bool(((x - w).abs() <= rel * w).all()) and bool((x != 0).any())
    assert bool(((c.float() - b.float()).abs() <= 2.0 ** -6 * 448).all())


@pytest.mark.parametrize("bounds", [(1, 6000), (40, 6000), (1, 300)])
def test_longer_than_max_kv_and_bad_lengths(mx, bounds):  # noqa: F811
    """Sequences past the stated limit, past the table and of negative length: NaN, and no weight of theirs written."""
    table, start, lens, pages = batch([2, 2, 2, 2], [100, 200, 50, 290], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(8, 4, 5)
    lens[1], lens[2] = 1 << 20, -3
    long = bounds[1] >= 6000
    lens[3] = 6001 if long else 301  # (of a table of fewer pages, or within it)
    before = torch.rand((pages, 2, 64), generator=torch.Generator().manual_seed(3))
    o, w = mx.cache_attend_weights(q, *cache, table.cuda(), ints(start), ints(lens), before.cuda(), True, *bounds)
    assert bool(o[:2].isfinite().all()) and bool(o[2:].isnan().all())
    t = torch.arange(102)
    used = torch.zeros(w.shape, dtype=torch.bool)
    used[table[0][t // 64].long(), :, t % 64] = True
    assert torch.equal(w.cpu()[~used], before[~used]) and bool((w.cpu()[used] != before[used]).any())


@pytest.mark.parametrize("new", [1, 6, 70])
def test_masked_nan_infinite_keys_and_lost_pages(mx, new):  # noqa: F811
    """What lies behind the end reaches nothing; a NaN query and a lost page make the weights of the keys that it sees
    NaN, and no others."""
    page, past = 64, 145
    table, start, lens, pages = batch([new, 1], [past, 10], page, spare=1)
    cache = filled(mx, pages, 2, page, 3)
    q = rows(new + 1, 6, 4)
    clean = mx.cache_attend_weights(q, *cache, table.cuda(), ints(start), ints(lens))
    kc, ks, vc, vs = (c.clone() for c in cache)
    L = lens[0]
    K, V = kc.view(pages, 2, page // 32, 8, 32, 16).transpose(3, 4), vc.transpose(3, 4)
    for t in range(L, -(-L // 32) * 32):
        K[int(table[0, t // page]), :, t % page // 32, t % 32] = 0x7F
        V[int(table[0, t // page]), :, t % page // 32, t % 32] = 0x7F
    got = mx.cache_attend_weights(q, kc, ks, vc, vs, table.cuda(), ints(start), ints(lens))
    assert all(torch.equal(a, b) for a, b in zip(clean, got))
    bad = q.clone()
    bad[0, 0] = math.nan  # token 0, head 0 of group 0: it sees keys up to `past`
    w = mx.cache_attend_weights(bad, *cache, table.cuda(), ints(start), ints(lens))[1].cpu()
    x = steps.weights_of(w, table[0], L, 0)
    assert bool(x[:past + 1].isnan().all()) and bool(x[past + 1:].isfinite().all())
    assert bool(steps.weights_of(w, table[0], L, 1).isfinite().all())
    assert bool(steps.weights_of(w, table[1], lens[1], 0).isfinite().all())
    lost = table.clone()
    lost[0, 1] = pages
    o, w = mx.cache_attend_weights(q, *cache, lost.cuda(), ints(start), ints(lens))
    assert bool(o[:new].isnan().all()) and bool(o[new:].isfinite().all())
    x = steps.weights_of(w.cpu(), table[0], L, 0)
    assert bool(x[:64].isnan().all()) and bool((x[64:128] == 0).all()) and bool(x[128:].isnan().all())


def test_weights_in_a_graph_and_on_a_stream(mx):  # noqa: F811
    table, start, lens, pages = batch([1, 1, 3], [3000, 10, 5000], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(5, 8, 5)
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    for bounds in ((3, 5003), (64, 5003)):
        w = torch.zeros((pages, 2, 64), device="cuda")
        mx.cache_attend_weights(*args, w, True, *bounds)
        step = w.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            mx.cache_attend_weights(*args, w, True, *bounds)
        w.zero_()
        for i in range(3):  # the weights of the keys that were there add up
            g.replay()
            torch.cuda.synchronize()
            new = [table[s, (lens[s] - 1) // 64] for s in range(2)]
            p, o = int(new[0]), (lens[0] - 1) % 64
            assert torch.equal(w[p, :, o], step[p, :, o])
            p = int(table[0, 0])
            assert torch.allclose(w[p], (i + 1) * step[p], rtol=2.0 ** -21, atol=0)
            mx.cache_attend(*args)
        s = torch.cuda.Stream()
        v = torch.zeros_like(w)
        s.wait_stream(torch.cuda.current_stream())
        mx.cache_attend_weights(*args, v, True, *bounds, stream=s)
        s.synchronize()
        assert torch.equal(v, step)
