"""Rotation by position in a cache that was cut: kept keys keep theirs, new ones are given theirs."""
import pytest

import cache_reference as ref
from test_gpu_cache import batch, ints, mx, rows  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
@pytest.mark.parametrize("in_place", [False, True])
def test_keys_after_a_cut_keep_their_positions(mx, in_place, pairs):  # noqa: F811
    """Two prompts are cut to a budget and go on by three tokens each.  Every key of the cache is then the one that was
    projected, turned by its position without the cut.

    Tolerance: a key is rounded to E4M3 once by half a step, 2^-4 of itself or 2^-10 of its block's scale; each of the
    roundings of a block that grows (compaction, three appends) moves it by 2^-10 of a scale at most, and by none where
    it is above 2^-6 of it; fp32 rotation adds 2^-20 of the pair."""
    H, page, budget = 2, 32, 70
    lens = [150, 93]
    table, start, lens, pages = batch(lens, [0, 0], page, spare=0)
    cache = tuple(torch.zeros(x, dtype=torch.uint8, device="cuda") for x in mx.cache_shapes(pages + 6, H, page))
    cos, sin = ref.tables(200, 128)
    tables = (cos.cuda(), sin.cuda())
    k, v = rows(start[-1], H, 1), rows(start[-1], H, 2)
    mx.cache_append(k, v, *cache, table.cuda(), ints(start), ints(lens), None, 1e-6, *tables, pairs=pairs)
    w = torch.rand((pages + 6, H, page), generator=torch.Generator().manual_seed(1))
    kept, counts = mx.cache_select(w.cuda(), table.cuda(), ints(lens), budget, 4, 9)
    out = table if in_place else torch.arange(6, dtype=torch.int32).view(2, 3) + pages
    mx.cache_compact(*cache, table.cuda(), kept, counts, None, None if in_place else out.cuda())
    kept = kept.cpu()
    keys = [[(k[start[s]:start[s + 1], h].cpu()[kept[s, h].long()], kept[s, h]) for h in range(H)] for s in range(2)]
    table, at = out.cuda(), counts.tolist()
    for i in range(3):
        at = [n + 1 for n in at]
        k, v = rows(2, H, 10 + i), rows(2, H, 20 + i)
        mx.cache_append(k, v, *cache, table, ints([0, 1, 2]), ints(at), None, 1e-6, *tables, ints([n + i for n in lens]), pairs)
        keys = [[(torch.cat((keys[s][h][0], k[s:s + 1, h].cpu())), torch.cat((keys[s][h][1], torch.tensor([lens[s] + i]))))
                 for h in range(H)] for s in range(2)]
    c = ref.Cache(*cache)
    for s in range(2):
        for h in range(H):
            x, pos = keys[s][h]
            want, size = ref.turned(x, None, 0.0, cos[pos.long()], sin[pos.long()], pairs)
            t = torch.arange(len(pos))
            scale = torch.exp2(c.ke[out[s, t // page].long(), h, t % page // 32].double())[:, None]
            err = (c.rows(out[s], len(pos), h)[0] - want).abs()
            tol = 2.0 ** -4 * want.abs() + 5 * 2.0 ** -10 * scale + 2.0 ** -20 * size
            assert bool((err <= tol).all())
            place = t  # turned by their place, the keys behind the first few would be others
            other = ref.turned(x, None, 0.0, cos[place], sin[place], pairs)[0]
            assert bool(((c.rows(out[s], len(pos), h)[0] - other).abs() > tol).any(-1)[-3:].all())
