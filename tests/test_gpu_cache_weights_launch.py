"""Weights of keys for as many sequences and heads as the call takes: more than one dimension of a launch holds with
workgroups of 512 threads."""
import pytest

import cache_reference as ref
import cache_steps_reference as steps
import cache_weights_check as check
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("S,H", [((1 << 20) - 1, 8), (1 << 20, 8), ((1 << 20) - 3, 15)])
def test_millions_of_heads(mx, S, H):  # noqa: F811
    """Up to 2^20 sequences (the most) of 8 and 15 heads, around and above 2^23 items, of which four sequences have
    tokens: the first, the last, and two between."""
    page = 64
    at = [0, 77777, S // 2 + 1, S - 1]
    new, past = [130, 3, 1, 60], [20, 40, 0, 4]
    few, start4, lens4, pages = batch(new, past, page)
    cache = filled(mx, pages, H, page, 7)
    table = torch.full((S, few.shape[1]), -1, dtype=torch.int32)
    lens, counts = (torch.zeros(S, dtype=torch.int32) for _ in range(2))
    for i, s in enumerate(at):
        table[s], lens[s], counts[s] = few[i], lens4[i], new[i]
    start = torch.cat((torch.zeros(1, dtype=torch.int32), counts.cumsum(0).int())).cuda()
    q = rows(start4[-1], H, 5)
    sums = steps.attend(ref.Cache(*cache), q.cpu(), few, start4, lens4, steps.causal)[2]
    o, w = mx.cache_attend_weights(q, *cache, table.cuda(), start, lens.cuda(), None, True, 130, max(lens4))
    used = check.weights(w.cpu(), sums, None, few, start4, lens4)
    assert bool((w.cpu()[~used] == 0).all()) and bool(o.isfinite().all())
