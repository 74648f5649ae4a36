"""Outputs that the binding makes for a call on another stream than the current one."""
import pytest

import cache_steps_reference as steps
from test_gpu_cache import batch, filled, ints, mx, rows  # noqa: F401
from test_gpu_cache_evict import heavy

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_outputs_are_not_memory_that_the_current_stream_may_still_use(mx):  # noqa: F811
    """What the current stream's allocator has free belongs to work enqueued there: an output that another stream
    writes is none of it.  Then the results, and the memory is reused by calls on that stream once it is free."""
    S, H, page, budget = 64, 4, 64, 4096
    lens = [100 * i for i in range(S)]
    table, _, lens, pages = batch([0] * S, lens, page)
    w = heavy(pages, H, page, 5).cuda()
    t, L = table.cuda(), ints(lens)
    want, n = steps.select(w.cpu(), table, lens, budget, 4, 100)
    s = torch.cuda.Stream()
    free = [torch.empty((S, H, budget), dtype=torch.int32, device="cuda") for _ in range(3)]
    places = {x.data_ptr() for x in free}
    torch.cuda.synchronize()
    del free
    for stream in (s, s.cuda_stream):
        kept, counts = mx.cache_select(w, t, L, budget, 4, 100, stream=stream)
        s.synchronize()
        assert kept.data_ptr() not in places
        assert torch.equal(kept.cpu(), want) and counts.tolist() == n
    kept = mx.cache_select(w, t, L, budget, 4, 100)[0]  # (the current stream's is)
    assert kept.data_ptr() in places


def test_every_call_on_another_stream(mx):  # noqa: F811
    """Outputs of attention, selection, norm, quantizers and the forward on a stream that is given equal the current one's."""
    table, start, lens, pages = batch([1, 40], [300, 900], 64)
    cache = filled(mx, pages, 2, 64, 7)
    q = rows(start[-1], 8, 5)
    args = (q, *cache, table.cuda(), ints(start), ints(lens))
    tree = torch.full((start[-1], 2), -1, dtype=torch.int32, device="cuda")
    w = torch.rand((pages, 2, 64), device="cuda")
    x = rows(3 * 64, 128, 4).view(1, 3, 64 * 128, 128)[:, :, :64].contiguous()
    calls = [
        lambda **k: mx.cache_attend(*args, **k), lambda **k: mx.cache_attend_window(*args, 100, 4, **k),
        lambda **k: mx.cache_attend_tree(*args, tree, **k),
        lambda **k: mx.cache_attend_weights(*args, w, weights_out=torch.zeros_like(w) if not k else zeros, **k),
        lambda **k: mx.cache_select(w, args[5], args[7], 100, **k), lambda **k: mx.qk_norm_rope(x, x, **k),
        lambda **k: mx.quantize(x, mx.AXIS_TOKENS, "uos", **k), lambda **k: mx.forward(x, x, x, "uos_pnq", **k),
        lambda **k: mx.cross_forward(x, x, x, "uos_pnq", **k), lambda **k: mx.softmax_rows(x, x, **k),
        lambda **k: mx.qmax_sse(x, mx.AXIS_TOKENS, [7.25], **k),
    ]
    s = torch.cuda.Stream()
    for i, call in enumerate(calls):
        zeros = torch.zeros_like(w)
        want = call()
        torch.cuda.synchronize()
        got = call(stream=s)
        s.synchronize()
        pairs = zip(want, got) if isinstance(want, tuple) else [(want, got)]
        for a, b in pairs:
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), i
