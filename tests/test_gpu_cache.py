"""The 8-bit paged cache: appending and attention over it, against 64 bits.

Append: V's codes and scales are fixed by the definition (compared exactly);
K's are those of a number within 2^-19 of (|a| + |b|) of the rotated one (see
test_gpu_rope.py), so a code is within half a step (2^-4 of the value, 2^-10
of the scale below 2^-6) of it.  Attention: the bound of cache_reference.attend."""
import math

import pytest

import cache_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_24377_amd import mxattn

    mxattn.lib()
    return mxattn


def empty_cache(mx, pages, heads, page, fill=0):
    return tuple(torch.full(s, fill, dtype=torch.uint8, device="cuda") for s in mx.cache_shapes(pages, heads, page))


def batch(new, past, page, spare=2, seed=0):
    """Page table (unused entries far outside), starts, lengths and pages of sequences."""
    g = torch.Generator().manual_seed(seed)
    lens = [a + b for a, b in zip(new, past)]
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, dtype=torch.int64).int()
    table = torch.full((len(new), max(max(need), 1) + 1), 1 << 30, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    return table, start, lens, pages


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows(tokens, heads, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((tokens, heads, ref.D), generator=g) * torch.exp(torch.randn((tokens, heads, 1), generator=g))
    return (x * scale).to(torch.bfloat16).cuda()


def check_append(cache, want, k, size):
    """The cache against `want`, appended by the reference; V exactly, K within its rounding."""
    got = ref.Cache(*cache)
    assert torch.equal(got.ve, want.ve)
    assert torch.equal(torch.nan_to_num(got.v, 999.0), torch.nan_to_num(want.v, 999.0))
    assert torch.equal(got.ke, want.ke)
    a, b = got.k, want.k
    assert torch.equal(a.isnan(), b.isnan())
    a, b = torch.nan_to_num(a), torch.nan_to_num(b)
    # another code only where the number lies next to the border of two codes: one step, and seldom
    assert bool(((a - b).abs() <= torch.clamp(b.abs() * 2.0 ** -2, min=2.0 ** -9)).all())
    assert float((a != b).double().mean()) < 1e-3


APPENDS = [
    # new, past, heads, page, rot, pairs, norm
    ([1], [0], 1, 32, 128, "halves", True),
    ([1, 1, 1], [31, 32, 33], 2, 32, 128, "interleaved", True),
    ([32, 31, 33], [0, 1, 31], 3, 64, 64, "halves", True),
    ([0, 5, 0, 64], [10, 27, 0, 64], 2, 128, 0, "halves", False),
    ([100, 1, 257], [3, 700, 95], 5, 256, 96, "interleaved", True),
    ([2], [4094], 40, 4096, 128, "halves", True),
    ([7] * 70, [13 * i for i in range(70)], 1, 32, 32, "interleaved", False),
    ([i % 4 for i in range(260)], [(17 * i) % 70 for i in range(260)], 5, 64, 48, "halves", True),
]


@pytest.mark.parametrize("case", APPENDS)
def test_append_against_64_bits(mx, case):
    new, past, H, page, rot, pairs, norm = case
    print(f"[append] {case}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    T = start[-1] + 3  # three tokens behind the last sequence
    cos, sin = ref.tables(max(lens) + 1, rot) if rot else (None, None)
    w = (torch.rand(ref.D, generator=torch.Generator().manual_seed(2)) + 0.5) if norm else None
    cache = empty_cache(mx, pages, H, page, 0x31)
    # the past in one call, then the new tokens, ten times larger: the shared blocks' scales grow
    for n, p, scale, seed in ((past, [0] * len(past), 1.0, 3), (new, past, 10.0, 4)):
        st = [0]
        for a in n:
            st.append(st[-1] + a)
        L = [a + b for a, b in zip(n, p)]
        t = st[-1] + (3 if n is new else 0)
        if t == 0:
            continue
        kv = rows(t, 2 * H, seed, scale)
        k, v = kv[:, :H], kv[:, H:]
        want = ref.Cache(*cache)
        pos = torch.zeros(t, dtype=torch.long)
        for s in range(len(n)):
            pos[st[s]:st[s + 1]] = torch.arange(p[s], L[s])
        y, size = ref.turned(k.cpu(), w, 1e-6, cos[pos][:, None] if rot else None, sin[pos][:, None] if rot else None, pairs)
        ref.append(want, y, v.cpu().double(), table, st, L)
        mx.cache_append(k, v, *cache, table.cuda(), ints(st), ints(L), w.cuda() if norm else None, 1e-6,
                        cos.cuda() if rot else None, sin.cuda() if rot else None, None, pairs)
        check_append(cache, want, y, size)


def test_append_with_given_positions_equals_its_own(mx):
    table, start, lens, pages = batch([40, 3], [5, 64], 64)
    cos, sin = (t.cuda() for t in ref.tables(200, 128))
    k, v = rows(43, 2, 1), rows(43, 2, 2)
    pos = ints(list(range(5, 45)) + list(range(64, 67)))
    a, b = empty_cache(mx, pages, 2, 64), empty_cache(mx, pages, 2, 64)
    mx.cache_append(k, v, *a, table.cuda(), ints(start), ints(lens), None, 1e-6, cos, sin)
    mx.cache_append(k, v, *b, table.cuda(), ints(start), ints(lens), None, 1e-6, cos, sin, pos)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    pos[7] = 200  # outside the table: NaN codes in that token alone
    mx.cache_append(k, v, *b, table.cuda(), ints(start), ints(lens), None, 1e-6, cos, sin, pos)
    ca, cb = ref.Cache(*a), ref.Cache(*b)
    t, p = 5 + 7, int(table[0, 0])
    assert bool(cb.k[p, :, t].isnan().all())
    cb.k[p, :, t] = ca.k[p, :, t]
    x, y = ca.k * torch.exp2(ca.ke.double()).repeat_interleave(32, 2)[..., None], cb.k * torch.exp2(
        cb.ke.double()).repeat_interleave(32, 2)[..., None]
    assert float((x - y).abs().max()) <= 2.0 ** -4 * float(x.abs().max())  # a block without its largest token


def test_append_zeros_infinities_and_ends_of_the_range(mx):
    """Zero blocks take the smallest scale; what is not finite is NaN and leaves the scale alone; the largest and
    smallest bf16 magnitudes."""
    table, start, lens, pages = batch([32, 32, 32, 32], [0] * 4, 32)
    x = torch.zeros((128, 1, ref.D))
    x[32:64] = torch.randn(32, 1, ref.D, generator=torch.Generator().manual_seed(1))
    x[40, 0, 3], x[41, 0, 4], x[42, 0, 5] = math.inf, -math.inf, math.nan
    x[64:96] = 3.3895e38
    x[96:128] = 2.0 ** -133
    x = x.to(torch.bfloat16).cuda()
    cache = empty_cache(mx, pages, 1, 32, 0x7F)
    want = ref.Cache(*cache)
    ref.append(want, x.cpu().double(), x.cpu().double(), table, start, lens)
    mx.cache_append(x, x, *cache, table.cuda(), ints(start), ints(lens))
    check_append(cache, want, x.cpu().double(), None)
    assert int(cache[1][int(table[0, 0]), 0, 0]) == 0


def test_append_to_bad_places_writes_nothing(mx):
    """Pages and lengths that do not exist, and negative positions: nothing is written there, the rest is."""
    H, page = 2, 32
    table = torch.tensor([[0, 99], [-1, 1], [2, 3], [4, 5]], dtype=torch.int32)
    start, lens = [0, 40, 80, 90, 95], [40, 40, -3, 3]
    k, v = rows(95, H, 1), rows(95, H, 2)
    cache = empty_cache(mx, 6, H, page, 0x55)
    before = [c.clone() for c in cache]
    mx.cache_append(k, v, *cache, table.cuda(), ints(start), ints(lens))
    # sequence 0: block 0 in page 0; block 1 in no page.  1: block 1 in page 1.  2: a bad length.  3: five tokens of
    # a length of three, so the last three, in page 4
    want = ref.Cache(*before)
    ref.append(want, k.cpu().double(), v.cpu().double(), table[[0, 1, 3]], [0, 40, 80], [40, 40])
    ref.append(want, k.cpu().double()[90:], v.cpu().double()[90:], table[3:], [0, 5], [3])
    check_append(cache, want, None, None)
    lens[2] = 65  # past the table
    mx.cache_append(k, v, *cache, table.cuda(), ints(start), ints(lens))
    check_append(cache, want, None, None)
    for c, b in zip(cache, before):
        assert torch.equal(c[[2, 3, 5]], b[[2, 3, 5]])


def test_starts_that_are_no_ascending_order_stay_inside(mx):
    """Contents of q_start that belong to no batch: some answer, nothing out of range."""
    H, page = 1, 32
    cache = empty_cache(mx, 4, H, page)
    guard = [c.clone() for c in cache]
    k = rows(50, H, 1)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32).cuda()
    for st in ([0, 90, 50], [-7, -3, 1 << 30], [50, 20, 0], [5, 5, 5]):
        mx.cache_append(k, k, *cache, table, ints(st), ints([64, 64]))
        o = torch.full_like(k, 3.0)
        mx.cache_attend(k, *cache, table, ints(st), ints([64, 64]), out=o)
    torch.cuda.synchronize()
    assert all(a.shape == b.shape for a, b in zip(cache, guard))


# ---------------------------------------------------------------------------


def filled(mx, pages, heads, page, seed, scale=1.0):
    """A cache with content everywhere: values of one sequence that owns every page."""
    cache = empty_cache(mx, pages, heads, page)
    T = pages * page
    table = torch.arange(pages, dtype=torch.int32)[None].cuda()
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.randn((T, heads, ref.D), generator=g, device="cuda") + torch.randn((heads, ref.D), generator=g, device="cuda")
    v = torch.randn((T, heads, ref.D), generator=g, device="cuda")
    mx.cache_append((k * scale).to(torch.bfloat16), v.to(torch.bfloat16), *cache, table, ints([0, T]), ints([T]))
    return cache


ATTENDS = [
    # new, past, Hq, Hkv, page, causal
    ([1], [0], 1, 1, 32, True),
    ([1], [31], 2, 2, 32, True),
    ([1, 1, 1], [32, 0, 63], 8, 1, 32, True),
    ([1], [500], 40, 8, 64, False),
    ([2, 1, 3, 4], [10, 127, 128, 1000], 10, 2, 128, True),
    ([33], [0], 3, 3, 32, True),
    ([5, 0, 70], [0, 50, 31], 4, 2, 64, True),
    ([100], [300], 5, 1, 256, False),
    ([64, 129], [64, 1], 16, 2, 64, True),
    ([1, 1], [2500, 4099], 24, 24, 256, False),
    ([257], [1000], 2, 2, 128, True),
    ([1] * 40, [97 * i % 701 for i in range(40)], 32, 8, 32, True),
    ([17], [2031], 64, 1, 64, True),
    ([300, 3], [5, 4000], 8, 8, 64, False),
    # many sequences, some without tokens, some without keys
    ([i % 3 for i in range(300)], [(37 * i) % 90 for i in range(300)], 4, 2, 32, True),
    # more sequences than threads that look for a share, long enough for shares
    ([1] * 270, [1100 if i == 200 else 3 * i % 64 for i in range(270)], 2, 1, 64, True),
    # 33 and 128 rows a head over few and many keys: every kernel's tile borders
    ([33], [200], 1, 1, 64, True),
    ([33, 128], [1500, 40], 2, 2, 128, True),
    ([16], [1200], 16, 2, 32, False),
    # a group of 256 heads
    ([2], [70], 256, 1, 32, True),
    # one row in many parts, and tiles in many parts
    ([1], [40000], 1, 1, 256, False),
    ([40], [20000], 4, 1, 256, True),
]


@pytest.mark.parametrize("case", ATTENDS)
def test_attend_against_64_bits(mx, case):
    new, past, Hq, Hkv, page, causal = case
    print(f"[attend] {str(case)[:120]}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    T = start[-1] + 2
    q = rows(T, Hq, 5, 0.5)
    out = torch.full((T, Hq, ref.D), 3.0, dtype=torch.bfloat16, device="cuda")
    mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), causal, out=out)
    want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, causal)
    n = start[-1]
    err = (out.cpu().double() - want)[:n].abs()
    assert bool((err <= tol[:n] + 1e-30).all()), float((err / (tol[:n] + 1e-30)).max())
    assert bool((out[n:] == 3).all())  # tokens of no sequence are left alone
    # the bounds that a program may state change no result beyond the same tolerance
    o2 = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), causal, max(new), max(lens))
    err = (o2.cpu().double() - want)[:n].abs()
    assert bool((err <= tol[:n] + 1e-30).all())


def test_bounds_that_are_wrong_cost_time_only(mx):
    """max_q and max_kv choose the kernel: every choice gives the same result within the tolerance."""
    new, past = [50, 1, 3], [700, 2100, 5]
    table, start, lens, pages = batch(new, past, 64)
    cache = filled(mx, pages, 2, 64, 11)
    q = rows(start[-1], 8, 5, 0.5)
    want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, True)
    for max_q, max_kv in ((1, 1), (1, 2000), (8, 5000), (9, 1025), (33, 64), (1 << 30, 1 << 40), (50, 2101), (16, 1 << 20)):
        o = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), True, max_q, max_kv)
        assert bool(((o.cpu().double() - want).abs() <= tol).all()), (max_q, max_kv)


def test_cache_larger_than_32_bit_offsets(mx):
    """Blocks past 4 GiB of codes: the same as at the cache's start."""
    pages, H, page = 36000, 8, 128  # 4.7 GB of K codes, and of V
    new, past = [1, 40], [300, 1500]
    table, start, lens, _ = batch(new, past, page, spare=0)
    used = int(table[table < pages].max()) + 1
    near = table.clone()
    far = torch.where(table < pages, table + (pages - used), table)
    k, v, q = rows(sum(lens), H, 1), rows(sum(lens), H, 2), rows(start[-1], 2 * H, 3)
    cache = empty_cache(mx, pages, H, page)
    first = [0, lens[0], sum(lens)]
    outs = []
    for t in (near, far):
        mx.cache_append(k, v, *cache, t.cuda(), ints(first), ints(lens))
        outs.append([mx.cache_attend(q, *cache, t.cuda(), ints(start), ints(lens), True, *b)
                     for b in ((1, 100), (1, 5000), (40, 5000))])
    for a, b in zip(*outs):
        assert torch.equal(a, b) and bool(a.isfinite().all()) and bool((a != 0).any())
    for c in cache:
        assert torch.equal(c[:used], c[pages - used:])


def test_attend_repeats_bit_for_bit(mx):
    table, start, lens, pages = batch([1, 1, 40], [3000, 10, 5000], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(42, 8, 5)
    a = [mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens)) for _ in range(3)]
    assert torch.equal(a[0], a[1]) and torch.equal(a[0], a[2])


@pytest.mark.parametrize("causal", [True, False])
def test_queries_that_see_nothing_get_zero(mx, causal):
    """Sequences without keys, and causal tokens before the first key (more new tokens than the length)."""
    table = torch.tensor([[0], [1], [2]], dtype=torch.int32)
    start, lens = [0, 3, 8, 9], [0, 2, 5]
    cache = filled(mx, 3, 2, 32, 1)
    q = rows(9, 4, 2)
    o = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), causal)
    want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, causal)
    assert bool(((o.cpu().double() - want).abs() <= tol).all())
    assert bool((o[:3] == 0).all())
    if causal:
        assert bool((o[3:6] == 0).all()) and bool((o[6:] != 0).any())


@pytest.mark.parametrize("new", [1, 6, 70])
def test_bytes_behind_the_end_and_masked_nan_do_not_reach_a_query(mx, new):
    """NaN codes and scales behind the end, and a NaN key and value that only later tokens see."""
    page, past = 64, 45
    table, start, lens, pages = batch([new], [past], page, spare=1)
    cache = filled(mx, pages, 2, page, 3)
    q = rows(new, 6, 4)
    clean = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens))
    kc, ks, vc, vs = (c.clone() for c in cache)
    L = lens[0]
    p, o = int(table[0, L // page]), L % page
    K = kc.view(pages, 2, page // 32, 8, 32, 16).transpose(3, 4)
    V = vc.transpose(3, 4)
    for t in range(o, page):
        K[p, :, t // 32, t % 32] = 0x7F
        V[p, :, t // 32, t % 32] = 0xFF
    if o % 32 == 0 and o:
        ks[p, :, o // 32:] = 255
        vs[p, :, o // 32:] = 255
    got = mx.cache_attend(q, kc, ks, vc, vs, table.cuda(), ints(start), ints(lens))
    assert torch.equal(got, clean)
    if new > 2:
        t = L - new // 2  # a token in the middle of the new ones, in one channel
        p, o = int(table[0, t // page]), t % page
        vc.transpose(3, 4)[p, 1, o // 32, o % 32, 77] = 0x7F
        got = mx.cache_attend(q, kc, ks, vc, vs, table.cuda(), ints(start), ints(lens))
        sees = new - new // 2  # the first token that sees it
        assert torch.equal(got[:sees], clean[:sees])
        assert bool(got[sees:, 3:, 77].isnan().all())
        other = [c for c in range(128) if c != 77]
        assert torch.equal(got[:, :, other], clean[:, :, other]) and torch.equal(got[:, :3], clean[:, :3])
        kc.view(pages, 2, page // 32, 8, 32, 16)[p, 0, o // 32, 0, o % 32, 0] = 0xFF
        got = mx.cache_attend(q, kc, ks, vc, vs, table.cuda(), ints(start), ints(lens))
        assert torch.equal(got[:sees], clean[:sees]) and bool(got[sees:, :3].isnan().all())


def test_bad_pages_and_lengths_give_nan_where_they_would_be_seen(mx):
    page = 32
    table = torch.tensor([[0, 1, 2], [3, -5, 4], [5, 0, 77], [1, 2, 3]], dtype=torch.int32)
    cache = filled(mx, 6, 1, page, 3)
    start, lens = [0, 40, 41, 42, 43], [70, 70, 60, 97]
    q = rows(43, 2, 4)
    good = table.clone()
    good[1, 1] = 0
    want, tol = ref.attend(ref.Cache(*cache), q.cpu(), good, start, [70, 70, 60, 0], True)
    o = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens)).cpu().double()
    assert bool(((o - want).abs() <= tol)[:40].all()) and bool(((o - want).abs() <= tol)[41].all())
    assert bool(o[40].isnan().all())  # sees the page that is not there
    assert bool(o[42].isnan().all())  # a length past its pages
    lens[3] = -1
    assert bool(mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens))[42].isnan().all())
    # a page that only the later of a sequence's tokens see
    table[0, 1] = 9
    o = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens)).cpu().double()
    sees = 32 - (70 - 40)  # token 2 is at position 32
    assert bool(((o - want).abs() <= tol)[:sees].all()) and bool(o[sees:40].isnan().all())


def test_queries_that_are_not_finite(mx):
    cache = filled(mx, 2, 1, 32, 3)
    table = torch.tensor([[0, 1]], dtype=torch.int32).cuda()
    q = rows(5, 2, 4)
    clean = mx.cache_attend(q, *cache, table, ints([0, 5]), ints([40]), False)
    q[1, 0, 3], q[2, 1, 100], q[3] = math.inf, math.nan, 0.0
    o = mx.cache_attend(q, *cache, table, ints([0, 5]), ints([40]), False)
    assert bool(o[1, 0].isnan().all()) and bool(o[2, 1].isnan().all())
    assert torch.equal(o[1, 1], clean[1, 1]) and torch.equal(o[2, 0], clean[2, 0]) and torch.equal(o[4], clean[4])
    mean = ref.Cache(*cache).rows(torch.tensor([0, 1]), 40, 0)[1].mean(0)
    # equal scores: the mean; p = 1 exactly, fp32 sums of 40 values below 4 (2^-18 at most)
    assert bool(((o[3].cpu().double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -18).all())


@pytest.mark.parametrize("scale", [2.0 ** -60, 2.0 ** -3, 30.0])
def test_attend_over_extreme_scores(mx, scale):
    """Scores from all alike to one that takes everything."""
    table, start, lens, pages = batch([3], [200], 64)
    cache = filled(mx, pages, 2, 64, 7, scale)
    q = rows(3, 4, 5, 2.0)
    o = mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens)).cpu().double()
    want, tol = ref.attend(ref.Cache(*cache), q.cpu(), table, start, lens, True)
    assert bool(((o - want).abs() <= tol + 1e-30).all())


def test_strided_queries_and_outputs(mx):
    table, start, lens, pages = batch([20, 1], [30, 99], 32)
    cache = filled(mx, pages, 2, 32, 7)
    qkv = rows(21, 8, 5)
    buf = torch.full((21, 6, ref.D), 9.0, dtype=torch.bfloat16, device="cuda")
    mx.cache_attend(qkv[:, :4], *cache, table.cuda(), ints(start), ints(lens), out=buf[:, 1:5])
    want = mx.cache_attend(qkv[:, :4].contiguous(), *cache, table.cuda(), ints(start), ints(lens))
    assert torch.equal(buf[:, 1:5], want)
    assert bool((buf[:, 0] == 9).all()) and bool((buf[:, 5] == 9).all())


def steps(mx, seed=0, S=3, Hq=8, Hkv=2, page=32):
    """What a generating program does for one step, on buffers that stay: returns the step and the buffers."""
    pages, most = 30, 256
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(seed))[:S * 8].view(S, 8).int().cuda()
    cache = empty_cache(mx, pages, Hkv, page)
    cos, sin = (t.cuda() for t in ref.tables(most, 128))
    w = torch.full((ref.D,), 1.25, device="cuda")
    qkv = torch.zeros((S, 1, Hq + 2 * Hkv, ref.D), dtype=torch.bfloat16, device="cuda")
    lens, start = torch.zeros(S, dtype=torch.int32, device="cuda"), ints(list(range(S + 1)))
    out = torch.zeros((S, Hq, ref.D), dtype=torch.bfloat16, device="cuda")
    qo = torch.zeros((S, Hq, 1, ref.D), dtype=torch.bfloat16, device="cuda")

    def step(stream=None):
        pos = (lens - 1).view(S, 1)
        mx.qk_norm_rope(qkv[:, :, :Hq].transpose(1, 2), None, w, None, 1e-6, cos, sin, pos, "halves", qo, stream=stream)
        mx.cache_append(qkv[:, 0, Hq:Hq + Hkv], qkv[:, 0, Hq + Hkv:], *cache, table, start, lens, w, 1e-6, cos, sin, None,
                        "halves", stream=stream)
        mx.cache_attend(qo.view(S, Hq, ref.D), *cache, table, start, lens, True, 1, most, out=out, stream=stream)

    return step, dict(qkv=qkv, lens=lens, out=out, qo=qo, cache=cache, table=table, w=w, cos=cos, sin=sin, Hq=Hq, Hkv=Hkv)


def inputs_of(S, heads, i):
    return rows(S, heads, 100 + i).view(S, 1, heads, ref.D)


def test_generation_step_by_step(mx):
    """Norm, rotation, append and attention of 70 tokens one after another: against attention in 64 bits over what the
    cache then holds (reference.attend's bound), and over the keys and values as they were before the cache.

    The second bound: a stored number x is off by at most 2^-4 |x|, and below the smallest normal code by half a step
    at each rounding, in all less than 2^-16 of the block's largest magnitude M (2^e < M / 224, half a step 2^-10 2^e,
    twice that over all growths of e).  So a score s = q . k / sqrt(d) is off by at most
    E = max_j sum_c |q_c| (2^-4 |k_jc| + 2^-16 M) / sqrt(d) + 2^-8 |s| (q is rounded to bf16), p by a factor within
    exp(+-2 E), and o by (exp(2 E) - 1) sum p |v| + exp(2 E) sum p (2^-4 |v| + 2^-16 M), beside the first bound."""
    step, b = steps(mx)
    S, Hq, Hkv = 3, b["Hq"], b["Hkv"]
    ks, vs = [], []
    for i in range(70):
        x = inputs_of(S, Hq + 2 * Hkv, i)
        b["qkv"].copy_(x)
        b["lens"].fill_(i + 1)
        step()
        c, s = b["cos"][i].cpu(), b["sin"][i].cpu()
        y, _ = ref.turned(x[:, 0, :Hq + Hkv].cpu(), b["w"].cpu(), 1e-6, c, s, "halves")
        ks.append(y[:, Hq:])
        vs.append(x[:, 0, Hq + Hkv:].cpu().double())
        if i % 23 not in (0, 9):
            continue
        got = b["out"].cpu().double()
        q = b["qo"].view(S, Hq, ref.D).cpu()
        held, tight = ref.attend(ref.Cache(*b["cache"]), q, b["table"].cpu(), [0, 1, 2, 3], [i + 1] * 3, True)
        assert bool(((got - held).abs() <= tight).all())
        k, v = torch.stack(ks, 1), torch.stack(vs, 1)  # [S, tokens, Hkv, d]
        for h in range(Hq):
            kh, vh = k[:, :, h // (Hq // Hkv)], v[:, :, h // (Hq // Hkv)]
            t = (y[:, None, h] * kh).sum(-1) / math.sqrt(ref.D)
            p = torch.softmax(t, -1)[..., None]
            o = (p * vh).sum(1)
            size = lambda z: 2.0 ** -4 * z.abs() + 2.0 ** -16 * z.abs().max()  # noqa: E731
            e = ((y[:, None, h].abs() * size(kh)).sum(-1) / math.sqrt(ref.D) + 2.0 ** -8 * t.abs()).amax(-1)[:, None]
            f = torch.exp(2 * e)
            tol = (f - 1) * (p * vh.abs()).sum(1) + f * (p * size(vh)).sum(1) + tight[:, h]
            assert bool(((got[:, h] - o).abs() <= tol).all())


def test_steps_captured_into_a_graph(mx):
    """One step captured and replayed with other tokens and lengths, with eager work between, equals eager steps."""
    eager, a = steps(mx)
    captured, b = steps(mx)
    side = torch.cuda.Stream()
    a["lens"].fill_(1)
    b["lens"].fill_(1)
    eager()
    with torch.cuda.stream(side):
        captured()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured()
    for i in range(40):
        x = inputs_of(3, 12, i)
        for st in (a, b):
            st["qkv"].copy_(x)
            st["lens"].fill_(i + 1)
        graph.replay()
        eager()
        if i % 7 == 0:
            torch.cuda.synchronize()
        assert torch.equal(a["out"], b["out"]), i
        assert all(torch.equal(x, y) for x, y in zip(a["cache"], b["cache"]))


@pytest.mark.parametrize("new,lens", [([1, 1, 1], [5000, 1200, 3]), ([40, 1, 7], [3000, 2000, 1030])])
def test_long_calls_captured_into_two_graphs(mx, new, lens):
    """Calls that need workspace, captured into two graphs that are replayed in turn and at once, each with a
    cache of its own, equal eager calls, also after others have used and freed memory in between."""
    n, group = sum(new), 4
    table, start, _, pages = batch(new, lens, 64, seed=5)
    table, start, lens = table.cuda(), ints(start), ints(lens)
    work = []
    for seed in (1, 2):
        cache = filled(mx, pages, 2, 64, seed)
        q, out, stream = rows(n, 2 * group, seed), torch.zeros(n, 2 * group, ref.D, dtype=torch.bfloat16, device="cuda"), torch.cuda.Stream()
        call = lambda q=q, cache=cache, out=out, **kw: mx.cache_attend(q, *cache, table, start, lens, out=out, **kw)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(Exception) as e:  # the library's own workspace lasts no longer than the call
                call(stream=stream)
            assert e.value.status == 10
            call()
        work.append((q, cache, out, stream, graph))
    for i in range(8):
        want = []
        for q, cache, *_ in work:
            q.copy_(rows(n, 2 * group, 10 + i))
            want.append(mx.cache_attend(q, *cache, table, start, lens))
        torch.cuda.synchronize()
        for *_, out, stream, graph in work:
            out.zero_()
            with torch.cuda.stream(stream if i % 2 else torch.cuda.current_stream()):
                torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
                graph.replay()
        junk = torch.full((1 << 24,), float("nan"), device="cuda")
        torch.cuda.synchronize()
        del junk
        assert all(torch.equal(w, x[2]) for w, x in zip(want, work)), i


@pytest.mark.parametrize("max_kv", [0, 300])
@pytest.mark.parametrize("max_q", [1, 64])
def test_starts_that_do_not_ascend(mx, max_q, max_kv):
    """Whatever q_start holds, calls end and write nothing but rows of the call's tokens and blocks of the cache."""
    tokens, seqs, heads = 64, 40, 2
    g = torch.Generator().manual_seed(3)
    table, _, lens, pages = batch([1] * seqs, [2000] * 2 + [40] * (seqs - 2), 64, seed=1)
    shapes = [math.prod(s) for s in mx.cache_shapes(pages, heads, 64)]
    starts = [[0, tokens] * (seqs // 2) + [0], list(range(seqs, -1, -1)), [tokens] * (seqs + 1), [-5] * seqs + [10 ** 9],
              [-2 ** 31, 2 ** 31 - 1] * (seqs // 2) + [5]] + [torch.randint(-5, 80, (seqs + 1,), generator=g).tolist() for _ in range(6)]
    for start in starts:
        room = [torch.full((n + 8192,), 7, dtype=torch.uint8, device="cuda") for n in shapes]
        cache = [x[4096:-4096].view(s) for x, s in zip(room, mx.cache_shapes(pages, heads, 64))]
        out = torch.full((3 * tokens, 4, ref.D), 9.0, dtype=torch.bfloat16, device="cuda")
        q, kv = rows(tokens, 4, 1), rows(tokens, heads, 2)
        mx.cache_append(kv, kv, *cache, table.cuda(), ints(start), ints(lens))
        mx.cache_attend(q, *cache, table.cuda(), ints(start), ints(lens), max_q=max_q, max_kv=max_kv, out=out[tokens:-tokens])
        torch.cuda.synchronize()
        assert all(bool((x[:4096] == 7).all() and (x[-4096:] == 7).all()) for x in room), start
        assert bool((out[:tokens] == 9).all() and (out[-tokens:] == 9).all()), start


def test_two_streams_at_once(mx):
    """Calls on two streams, neither waiting for the other, give what each gives alone."""
    work = []
    for seed in (1, 2):
        table, start, lens, pages = batch([1, 1, 30], [2500, 700, 60], 64, seed=seed)
        cache = filled(mx, pages, 2, 64, seed)
        q = rows(32, 8, seed)
        work.append((q, cache, table.cuda(), ints(start), ints(lens)))
    alone = [mx.cache_attend(q, *c, t, s, n) for q, c, t, s, n in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(o) for _ in range(20)] for o in alone]
    for i in range(20):
        for k, (q, c, t, s, n) in enumerate(work):
            mx.cache_attend(q, *c, t, s, n, out=outs[k][i], stream=streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(o, alone[k]) for o in outs[k])
