"""Attention that weighs the cache's keys against 64 bits, by every kernel: each weight a number, and within the bound
of the scores that all of them sum over."""
import pytest

import cache_reference as ref
import cache_steps_reference as steps
import cache_weights_check as check
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401
from test_gpu_cache_weights import WEIGHTS

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("scale", [0.5, 20.0])
@pytest.mark.parametrize("case", WEIGHTS)
def test_weights_are_numbers_within_the_bound(mx, case, scale):  # noqa: F811
    new, past, Hq, Hkv, page, causal = case
    print(f"[numbers] {str(case)[:120]} {scale}", flush=True)
    table, start, lens, pages = batch(new, past, page)
    cache = filled(mx, pages, Hkv, page, 7)
    q = rows(start[-1] + 2, Hq, 5, scale)
    before = torch.rand((pages, Hkv, page), generator=torch.Generator().manual_seed(3)) * 3
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.causal if causal else steps.everything)[2]
    for bounds in ((0, 0), (max(new), max(lens)), (1, max(lens)), (33, max(lens)), (129, 30000)):
        w = mx.cache_attend_weights(*args, before.cuda(), causal, *bounds, weights_out=torch.full_like(before, -7.0, device="cuda"))[1]
        used = check.weights(w.cpu(), sums, before, table, start, lens)
        assert bool((w.cpu()[~used] == -7).all())
    w = mx.cache_attend_weights(*args, None, causal)[1]
    check.weights(w.cpu(), sums, None, table, start, lens)


def test_many_short_sequences_and_their_scores_twice(mx):  # noqa: F811
    """20000 sequences of up to 32 keys, scores kept and (of a wide table, more than 1 GiB of them) computed again."""
    S = 20000
    t = torch.arange(S, dtype=torch.int32).view(S, 1)
    cache = filled(mx, S, 1, 32, 3)
    lens = [1 + 7 * i % 32 for i in range(S)]
    q = rows(S, 16, 6)
    some = list(range(0, S, 401)) + [S - 1]
    few = [lens[i] for i in some]
    sums = steps.attend(ref.Cache(*cache), q.cpu()[some], t[some], list(range(len(some) + 1)), few, steps.causal)[2]
    wide = torch.cat((t, torch.full((S, 31), -1, dtype=torch.int32)), 1)
    for table, m in ((t, 32), (wide, 1024)):
        w = mx.cache_attend_weights(q, *cache, table.cuda(), ints(list(range(S + 1))), ints(lens), None, True, 1, m)[1].cpu()
        check.weights(w, sums, None, t[some], list(range(len(some) + 1)), few)
        held = torch.arange(32) < torch.tensor(lens)[:, None]
        assert bool((w[:, 0][held] > 0).all()) and bool((w[:, 0][~held] == 0).all())


def test_outputs_of_many_short_sequences(mx):  # noqa: F811
    """The outputs beside those weights, of either way, within the bound of single outputs (a sample of sequences)."""
    S = 20000
    t = torch.arange(S, dtype=torch.int32).view(S, 1)
    cache = filled(mx, S, 1, 32, 3)
    lens = [1 + 7 * i % 32 for i in range(S)]
    q = rows(S, 16, 6)
    some = list(range(0, S, 97)) + [S - 1]
    want, tol, _ = steps.attend(ref.Cache(*cache), q.cpu()[some], t[some], list(range(len(some) + 1)), [lens[i] for i in some],
                                steps.causal)
    assert float(tol.max()) < 0.05 * float(want.abs().max())  # (a bound that could fail)
    wide = torch.cat((t, torch.full((S, 31), -1, dtype=torch.int32)), 1)
    for table, m in ((t, 32), (wide, 1024)):
        o = mx.cache_attend_weights(q, *cache, table.cuda(), ints(list(range(S + 1))), ints(lens), None, True, 1, m)[0].cpu()
        assert bool(o.isfinite().all())
        assert bool(((o[some].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("new,past,bounds", [([1, 3], [900, 500], (3, 903)), ([40, 60], [300, 1900], (60, 2000))])
@pytest.mark.parametrize("byte,power", [(0, 116), (0, 124), (1, 123), (20, 104)])
def test_keys_of_the_smallest_scales(mx, new, past, bounds, byte, power):  # noqa: F811
    """Scale bytes down to 0 (2^-127, which fp32 holds as a subnormal) under queries so large that scores count."""
    table, start, lens, pages = batch(new, past, 64)
    cache = filled(mx, pages, 2, 64, 7)
    cache[1].fill_(byte)
    q = (rows(start[-1], 8, 5).double().clamp(-3, 3) * 2.0 ** power).to(torch.bfloat16)
    want, tol, sums = steps.attend(ref.Cache(*cache), q.cpu(), table, start, lens, steps.causal)
    o, w = mx.cache_attend_weights(q, *cache, table.cuda(), ints(start), ints(lens), None, True, *bounds)
    assert bool(((o.cpu().double() - want).abs() <= tol).all())
    check.weights(w.cpu(), sums, None, table, start, lens)
