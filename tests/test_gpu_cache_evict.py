"""Selecting the tokens of a cache that stay, and moving them together: exact results, and a generation that uses both."""
import math

import pytest

import cache_reference as ref
import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def heavy(pages, heads, page, seed, kind="some"):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn((pages, heads, page), generator=g).mul_(2).exp_()
    if kind == "ties":
        w = torch.randint(0, 3, w.shape, generator=g).float()
    if kind == "equal":
        w = torch.full_like(w, 0.25)
    if kind == "even":
        w = torch.rand(w.shape, generator=g)
    if kind == "narrow":  # numbers next to one another
        w = 1 + torch.randint(0, 3000, w.shape, generator=g).float() * 2 ** -23
    if kind == "odd":  # zeros of both signs, negatives, infinities, NaN, subnormals
        pick = torch.randint(0, 8, w.shape, generator=g)
        for i, x in enumerate((0.0, -0.0, -1.5, math.inf, -math.inf, math.nan, 1e-40)):
            w[pick == i] = x
    return w


SELECTS = [
    # lengths, heads, page, budget, sinks, recent, weights
    ([1], 1, 32, 1, 0, 0, "some"),
    ([33], 2, 32, 1, 0, 0, "some"),
    ([0, 5, 100, 64], 3, 64, 64, 4, 10, "some"),
    ([300, 299, 17, 64, 65], 2, 32, 64, 0, 0, "ties"),
    ([1000, 4097], 2, 128, 500, 3, 100, "equal"),
    ([3000, 77], 5, 256, 200, 64, 64, "odd"),
    ([1025, 2048], 1, 64, 1024, 1024, 0, "some"),
    ([1025, 2048], 1, 64, 1024, 0, 1024, "some"),
    ([5000], 2, 32, 4999, 0, 1, "ties"),
    ([40000], 2, 256, 5000, 4, 1000, "some"),
    ([40000], 1, 4096, 39000, 0, 0, "ties"),
    ([90 * i % 1000 for i in range(200)], 2, 32, 128, 2, 30, "some"),
    # a table for more keys than a workgroup holds: several for each head, some of them without keys, whole
    # stretches that must stay, chunks of more than 4096 keys, more of a digit than the list takes
    ([17000, 40, 16384, 0, 8193], 3, 64, 3000, 5, 2000, "odd"),
    ([120000, 4097], 2, 256, 10000, 64, 1000, "some"),
    ([70000], 1, 32, 50000, 30000, 20000, "some"),
    ([70000], 1, 32, 50000, 30000, 19999, "some"),
    ([70000], 2, 64, 30000, 10, 20, "equal"),
    ([300000], 1, 1024, 100001, 0, 0, "ties"),
    ([300000], 1, 4096, 2, 0, 1, "odd"),
    ([300000, 65000, 9000], 2, 256, 90001, 4, 500, "even"),
    ([200000, 16385], 2, 128, 15000, 0, 0, "narrow"),
    # so many heads that each is one workgroup's, which reads its keys again in every pass
    ([20000, 16385, 30001] + [33 * i for i in range(127)], 2, 64, 3000, 4, 100, "odd"),
    ([20000, 16384, 65535] + [9 * i for i in range(61)], 4, 32, 20, 0, 0, "narrow"),
]


@pytest.mark.parametrize("case", SELECTS)
def test_select(mx, case):  # noqa: F811
    lens, H, page, budget, sinks, recent, kind = case
    print(f"[select] {str(case)[:120]}", flush=True)
    table, _, lens, pages = batch([0] * len(lens), lens, page)
    w = heavy(pages, H, page, 5, kind)
    kept, counts = mx.cache_select(w.cuda(), table.cuda(), ints(lens), budget, sinks, recent)
    want, n = steps.select(w, table, lens, budget, sinks, recent)
    assert counts.tolist() == n
    assert torch.equal(kept.cpu(), want)


def test_select_of_bad_lengths_and_pages(mx):  # noqa: F811
    table = torch.tensor([[0, 1], [2, 3], [4, 99], [1, 0]], dtype=torch.int32)
    w = heavy(6, 2, 32, 1)
    kept, counts = mx.cache_select(w.cuda(), table.cuda(), ints([-1, 65, 64, 64]), 40, 2, 3)
    assert counts.tolist() == [0, 0, 40, 40] and bool((kept[:2] == -1).all())
    lost = w.clone()
    lost[5] = math.nan  # the page that does not exist weighs as NaN
    t = torch.where(table == 99, 5, table)
    want, _ = steps.select(lost, t[2:], [64, 64], 40, 2, 3)
    assert torch.equal(kept[2:].cpu(), want)


def small_codes(cache, seed):
    """Scales that differ much from block to block, and codes down to the smallest: rounding at every shift."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    for s in (cache[1], cache[3]):
        s.copy_(torch.randint(120, 136, s.shape, generator=g, device="cuda").to(torch.uint8))
    for c in (cache[0], cache[2]):
        c.copy_(torch.randint(0, 256, c.shape, generator=g, device="cuda").to(torch.uint8))
    return cache


def check_cache(cache, want, w=None, ww=None):
    got = ref.Cache(*cache)
    assert torch.equal(got.ke, want.ke) and torch.equal(got.ve, want.ve)
    for a, b in ((got.k, want.k), (got.v, want.v)):
        assert torch.equal(a.isnan(), b.isnan())
        assert torch.equal(torch.nan_to_num(a, 999.0), torch.nan_to_num(b, 999.0))
    if w is not None:
        assert torch.equal(w.cpu(), ww)


COMPACTS = [
    # lengths, heads, page, budget, per head
    ([1], 1, 32, 1, True),
    ([33], 2, 32, 5, True),
    ([100, 64, 3, 70], 3, 64, 64, True),
    ([300, 299, 17, 64, 65], 2, 32, 200, True),
    ([1000, 700], 2, 128, 333, False),
    ([2000], 5, 256, 40, True),
    ([500, 600], 1, 4096, 499, True),
    ([9 * i % 150 for i in range(1, 60)], 2, 32, 70, True),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", COMPACTS)
def test_compact(mx, case, in_place):  # noqa: F811
    lens, H, page, budget, per_head = case
    print(f"[compact] {str(case)[:120]} {in_place}", flush=True)
    table, _, lens, pages = batch([0] * len(lens), lens, page)
    per = -(-budget // page)
    out = table if in_place else (torch.arange(len(lens) * per, dtype=torch.int32).view(-1, per) + pages)
    pages += 0 if in_place else out.numel()
    cache = small_codes(tuple(torch.empty(s, dtype=torch.uint8, device="cuda") for s in mx.cache_shapes(pages, H, page)), 3)
    w = heavy(pages, H, page, 5)
    kept, counts = steps.select(heavy(pages, H, page, 6), table, lens, budget, 0, 1)
    if not per_head:
        kept = kept[:, :1].contiguous()
    want, ww = ref.Cache(*cache), w.clone()
    steps.compact(want, table, out, kept, counts, [0] * len(lens), ww)
    wd = w.cuda()
    mx.cache_compact(*cache, table.cuda(), kept.cuda(), ints(counts), None, None if in_place else out.cuda(), wd)
    check_cache(cache, want, wd, ww)


@pytest.mark.parametrize("H", [1, 3])
def test_accepted_drafts_move_to_the_end(mx, H):  # noqa: F811
    """In place behind a base, the same tokens for all heads: none, some and all of them accepted; a base inside a
    block, at its end, at 0, and one whose tokens cross pages."""
    base = [45, 64, 0, 31, 200, 95, 10]
    accepted = [[46, 50, 61], [64, 65, 66], [3, 9], [], [203], list(range(96, 96 + 60, 2)), [10]]
    lens = [b + 64 for b in base]
    table, _, lens, pages = batch([0] * len(base), lens, 64)
    cache = small_codes(tuple(torch.empty(s, dtype=torch.uint8, device="cuda") for s in mx.cache_shapes(pages, H, 64)), 9)
    kept = torch.full((len(base), 1, 32), 1 << 30, dtype=torch.int32)
    for s, a in enumerate(accepted):
        kept[s, 0, :len(a)] = torch.tensor(a, dtype=torch.int32)
    counts = [len(a) for a in accepted]
    want = ref.Cache(*cache)
    steps.compact(want, table, table, kept, counts, base)
    t = table.cuda()
    mx.cache_compact(*cache, t, kept.cuda(), ints(counts), ints(base), t)  # (the table itself: in place)
    check_cache(cache, want)


def test_compact_of_bad_places(mx):  # noqa: F811
    """Positions and pages that do not exist and scales that are no number give NaN codes; counts and bases that do not
    fit, and pages to write that do not exist, leave all as it was."""
    page, H = 64, 2
    table = torch.tensor([[0, 1], [2, -5], [3, 4], [5, 6], [7, 8]], dtype=torch.int32)
    out = torch.tensor([[10], [11], [12], [13], [99]], dtype=torch.int32)
    cache = small_codes(tuple(torch.empty(s, dtype=torch.uint8, device="cuda") for s in mx.cache_shapes(14, H, page)), 4)
    cache[1][3, :, 1] = 255
    cache[3][3, 0, 0] = 255
    g = torch.Generator().manual_seed(2)
    kept = torch.stack([torch.stack([torch.randperm(128, generator=g)[:50] for _ in range(H)]) for _ in range(5)]).int()
    kept[0, 0, 7], kept[0, 1, 9], kept[0, 1, 10] = -1, 128, 1 << 30
    w = heavy(14, H, page, 5)
    for counts, base in (([50, 50, 50, 50, 50], [0, 3, 0, 14, 0]), ([51, -1, 0, 50, 50], [0, 0, 0, 15, -1])):
        want, ww, wd = ref.Cache(*cache), w.clone(), w.cuda()
        steps.compact(want, table, out, kept, counts, base, ww)
        mx.cache_compact(*cache, table.cuda(), kept.cuda(), ints(counts), ints(base), out.cuda(), wd)
        check_cache(cache, want, wd, ww)
        w = ww


def test_in_place_with_any_contents_stays_inside(mx):  # noqa: F811
    """kept that does not ascend: some contents, nothing out of range and nothing beside the sequence's pages."""
    table, _, lens, pages = batch([0, 0], [300, 200], 32)
    cache = filled(mx, pages, 2, 32, 7)
    before = [c.clone() for c in cache]
    kept = torch.randint(-5, 1 << 20, (2, 2, 150), generator=torch.Generator().manual_seed(2)).int()
    mx.cache_compact(*cache, table.cuda(), kept.cuda(), ints([150, 150]))
    free = [p for p in range(pages) if p not in table.tolist()[0] + table.tolist()[1]]
    for a, b in zip(cache, before):
        assert torch.equal(a[free], b[free])


def test_starts_and_lengths_that_belong_to_no_batch_stay_inside(mx):  # noqa: F811
    """q_start that does not ascend, lengths, counts and bases of any value: some answer, nothing out of range."""
    H, page, S = 2, 32, 4
    table = torch.arange(8, dtype=torch.int32).view(S, 2).cuda()
    cache = filled(mx, 10, H, page, 7)
    before = [c.clone() for c in cache]
    q = rows(50, 4, 1)
    tree = torch.full((50, 1), -1, dtype=torch.int32, device="cuda")
    w = torch.ones((10, H, page), device="cuda")
    for st in ([0, 90, 50, 20, 50], [-7, -3, 1 << 30, 0, 5], [50, 20, 0, 0, 0], [5, 5, 5, 5, 5]):
        for L in ([64, 64, 64, 64], [-1, 1 << 30, 65, 0], [3, 64, 1, 33]):
            batch_ = (q, *cache, table, ints(st), ints(L))
            for b in ((0, 0), (1, 64), (1, 5000), (50, 5000)):
                mx.cache_attend_window(*batch_, 20, 3, True, *b)
                mx.cache_attend_window(*batch_, 20, 3, False, *b)
                mx.cache_attend_tree(*batch_, tree, *b)
                mx.cache_attend_weights(*batch_, w, True, *b)
            kept, counts = mx.cache_select(w, table, ints(L), 30, 2, 5)
            mx.cache_compact(*cache, table, kept, ints(L), ints(st[:4]), weights=w)
            torch.cuda.synchronize()
    for c, b in zip(cache, before):  # pages of no sequence
        assert torch.equal(c[8:], b[8:])
    assert bool((w[8:] == 1).all())


def test_eviction_in_a_graph(mx):  # noqa: F811
    """Selection and compaction captured together and replayed with other weights."""
    lens, H, page, budget = [700, 90, 1200], 2, 64, 256
    table, _, lens, pages = batch([0] * 3, lens, page)
    out = torch.arange(12, dtype=torch.int32).view(3, 4) + pages
    cache = filled(mx, pages + 12, H, page, 7)
    w = torch.zeros((pages + 12, H, page), device="cuda")
    t, o, L = table.cuda(), out.cuda(), ints(lens)
    mx.cache_compact(*cache, t, *mx.cache_select(w, t, L, budget, 4, 32), None, o)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept, counts = mx.cache_select(w, t, L, budget, 4, 32)
        mx.cache_compact(*cache, t, kept, counts, None, o)
    for seed in range(3):
        x = heavy(pages + 12, H, page, seed)
        w.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        want, n = steps.select(x, table, lens, budget, 4, 32)
        assert torch.equal(kept.cpu(), want) and counts.tolist() == n
        c = ref.Cache(*cache)
        steps.compact(c, table, out, want, n, [0] * 3)
        check_cache(cache, c)


def test_steps_past_32_bit_offsets(mx):  # noqa: F811
    """Blocks past 4 GiB of codes: the same as at the cache's start."""
    pages, H, page = 36000, 8, 128  # 4.7 GB of K codes, and of V
    new, past = [1, 40], [300, 1500]
    table, start, lens, _ = batch(new, past, page, spare=0)
    table = torch.where(table < pages, table, -1)
    used = int(table.max()) + 1
    out = torch.arange(2 * 4, dtype=torch.int32).view(2, 4) + used  # 400 tokens each
    used += 8
    k, v, q = rows(sum(lens), H, 1), rows(sum(lens), H, 2), rows(start[-1], 2 * H, 3)
    cache = tuple(torch.zeros(s, dtype=torch.uint8, device="cuda") for s in mx.cache_shapes(pages, H, page))
    w = torch.zeros((pages, H, page), device="cuda")
    first = [0, lens[0], sum(lens)]
    tree = torch.full((start[-1], 2), -1, dtype=torch.int32, device="cuda")
    got = []
    for shift in (0, pages - used):
        t, o = torch.where(table >= 0, table + shift, table).cuda(), (out + shift).cuda()
        mx.cache_append(k, v, *cache, t, ints(first), ints(lens))
        args = (q, *cache, t, ints(start), ints(lens))
        res = [mx.cache_attend_window(*args, 700, 40, True, *b) for b in ((1, 100), (1, 5000), (40, 5000))]
        res += [mx.cache_attend_tree(*args, tree, *b) for b in ((1, 5000), (40, 5000))]
        res += [mx.cache_attend_weights(*args, w, True, *b)[0] for b in ((1, 1600), (40, 1600))]
        kept, counts = mx.cache_select(w, t, ints(lens), 400, 4, 20)
        mx.cache_compact(*cache, t, kept, counts, None, o, w)
        mx.cache_compact(*cache, t, kept, counts)
        got.append(res + [kept, counts] + [x[shift:shift + used].clone() for x in (*cache, w)])
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool((a != 0).any())


def test_two_graphs_one_after_another(mx):  # noqa: F811
    """Calls with workspace captured twice, on other inputs, and replayed in turn: neither uses the other's."""
    lens, H, page = [700, 2100], 2, 256
    table, _, lens, pages = batch([0] * 2, lens, page)
    table = torch.cat((torch.where(table < pages, table, -1), torch.full((2, 80), -1, dtype=torch.int32)), 1)  # > 16384 keys
    cache = filled(mx, pages, H, page, 7)
    t, L, st = table.cuda(), ints(lens), ints([0, 1, 2])
    calls, graphs, outs, want = [], [], [], []
    for i in range(2):
        q, w = rows(2, 8, 10 + i), heavy(pages, H, page, i).cuda()

        def call(q=q, w=w):
            o, v = mx.cache_attend_weights(q, *cache, t, st, L, w, True, 1, 2100, weights_out=torch.zeros_like(w))
            return [o, v, *mx.cache_select(v, t, L, 300, 2, 9),
                    mx.cache_attend_window(q, *cache, t, st, L, 1500, 3, True, 1, 2100)]
        want.append(call())
        calls.append(call)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    for i in (0, 1, 1, 0, 0, 1):
        for x in outs[i]:
            x.zero_()
        graphs[i].replay()
        calls[1 - i]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w))


def test_a_generation_with_drafts_and_eviction(mx):  # noqa: F811
    """Prompts are appended and weighed, cut to a budget in place, generation goes on with a window, a tree of drafts is
    verified and its accepted path stays: every attention agrees with 64 bits over what the cache holds."""
    H, Hq, page, budget = 2, 8, 32, 96
    lens = [150, 70, 200]
    table, start, lens, pages = batch(lens, [0, 0, 0], page, spare=3)
    table = torch.cat((torch.where(table < pages, table, torch.tensor(-1, dtype=torch.int32)),
                       torch.full((3, 2), -1, dtype=torch.int32)), 1)
    pages += 6
    table[:, -2:] = torch.arange(6, dtype=torch.int32).view(3, 2) + pages - 6
    for s in range(3):  # unused entries behind a sequence's pages: its spare ones
        used = -(-lens[s] // page)
        table[s, used:used + 2] = table[s, -2:].clone()
    cache = tuple(torch.zeros(x, dtype=torch.uint8, device="cuda") for x in mx.cache_shapes(pages, H, page))
    t = table.cuda()

    def attend_ok(o, q, start, lens, sees):
        want, tol, sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, sees)
        assert bool(((o.cpu().double() - want).abs() <= tol + 1e-30).all())
        return sums

    k, v, q = rows(start[-1], H, 1), rows(start[-1], H, 2), rows(start[-1], Hq, 3, 0.5)
    mx.cache_append(k, v, *cache, t, ints(start), ints(lens))
    w = torch.zeros((pages, H, page), device="cuda")
    o, _ = mx.cache_attend_weights(q, *cache, t, ints(start), ints(lens), w)
    attend_ok(o, q, start, lens, steps.causal)
    kept, counts = mx.cache_select(w, t, ints(lens), budget, 4, 20)
    assert torch.equal(kept.cpu(), steps.select(w.cpu(), table, lens, budget, 4, 20)[0])
    mx.cache_compact(*cache, t, kept, counts, weights=w)
    lens = counts.tolist()
    assert lens == [96, 70, 96]
    # two tokens more, seen through a window, and weighed
    one = [0, 1, 2, 3]
    for i in range(2):
        lens = [n + 1 for n in lens]
        k, v, q = rows(3, H, 10 + i), rows(3, H, 20 + i), rows(3, Hq, 30 + i, 0.5)
        mx.cache_append(k, v, *cache, t, ints(one), ints(lens))
        o = mx.cache_attend_window(q, *cache, t, ints(one), ints(lens), 50, 4)
        attend_ok(o, q, one, lens, steps.window(50, 4, True))
        mx.cache_attend_weights(q, *cache, t, ints(one), ints(lens), w)
    # drafts: a root, two children, a grandchild of the second
    mask = torch.tensor([[0b1], [0b11], [0b101], [0b1101]], dtype=torch.int32).repeat(3, 1)
    four, past = [0, 4, 8, 12], lens
    lens = [n + 4 for n in lens]
    k, v, q = rows(12, H, 40), rows(12, H, 41), rows(12, Hq, 42, 0.5)
    mx.cache_append(k, v, *cache, t, ints(four), ints(lens))
    o = mx.cache_attend_tree(q, *cache, t, ints(four), ints(lens), mask.cuda())
    attend_ok(o, q, four, lens, steps.tree(mask))
    accepted = [[0, 2, 3], [0, 1], [0]]
    kept = torch.zeros((3, 1, 4), dtype=torch.int32)
    for s, a in enumerate(accepted):
        kept[s, 0, :len(a)] = torch.tensor(a) + past[s]
    c = ref.Cache(*cache)
    before = [c.rows(table[s], lens[s], h) for s in range(3) for h in range(H)]
    step = 2.0 ** (max(int(c.ke.max()), int(c.ve.max())) - 9)  # of the smallest numbers of the largest scale
    mx.cache_compact(*cache, t, kept.cuda(), ints([3, 2, 1]), ints(past))
    for i, (kk, vv) in enumerate(before):
        s, h = divmod(i, H)
        n = past[s] + len(accepted[s])
        at = torch.cat((torch.arange(past[s]), torch.tensor(accepted[s]) + past[s]))
        for a, b in zip(ref.Cache(*cache).rows(table[s], n, h), (kk[at], vv[at])):
            assert bool(((a - b).abs() <= step / 2).all())  # exact, or rounded to a multiple of that
    lens = [p + len(a) for p, a in zip(past, accepted)]
    q = rows(3, Hq, 50, 0.5)
    o = mx.cache_attend(q, *cache, t, ints(one), ints(lens))
    attend_ok(o, q, one, lens, steps.causal)
