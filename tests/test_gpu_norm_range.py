"""The norm of heads over the whole range of bf16: squares that leave fp32's range in either direction.
Tolerances as in test_gpu_rope.py and test_gpu_cache.py."""
import math

import pytest

import cache_reference as ref
from test_gpu_cache import batch, check_append, empty_cache, ints, mx  # noqa: F401
from test_gpu_rope import _check, _heads

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

POWERS = [-126, -100, -76, -75, -64, -50, -48, -46, -44, 0, 58, 60, 62, 64, 100, 120]


def scaled(q, eps):
    """Row n of q [1, H, N, d] times 2^POWERS[n], and some rows that mix the ends."""
    for n, p in enumerate(POWERS):
        q[:, :, n] = (q[:, :, n].float() * 2.0 ** p).to(torch.bfloat16)
    q[:, 0, 0, ::2] = 2.0 ** -133          # the smallest magnitude
    q[:, 0, 1] = 0
    q[:, 0, 1, 7] = -2.0 ** -133            # alone
    q[:, 0, 14, ::3] = 3.3895e38            # the largest
    q[:, 0, 15, 1:] = 2.0 ** -133
    q[:, 0, 15, 0] = 3.3895e38              # both
    return q


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-30, 1e-6, 1e30, 2.9e38])
def test_norm_of_every_magnitude(mx, eps):  # noqa: F811
    print(f"[norm] eps {eps}", flush=True)
    q = scaled(_heads(1, 3, len(POWERS), "bhn", 11), eps)
    w = (torch.rand(ref.D, generator=torch.Generator().manual_seed(3)) + 0.5).cuda()
    o, _ = mx.qk_norm_rope(q, None, w, None, eps)
    e = float(torch.tensor(eps, dtype=torch.float32))  # as the call takes it
    assert bool(o.isfinite().all())
    _check(o, q, w, e, None, None, None, "halves")


def test_zero_rows_without_eps_are_no_numbers(mx):  # noqa: F811
    """0 / 0, as the formula has it; with the smallest eps, 0."""
    q = torch.zeros((1, 1, 2, ref.D), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(ref.D, device="cuda")
    assert bool(mx.qk_norm_rope(q, None, w, None, 0.0)[0].isnan().all())
    assert bool((mx.qk_norm_rope(q, None, w, None, 1e-45)[0] == 0).all())


@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_appended_keys_of_every_magnitude(mx, eps):  # noqa: F811
    n = len(POWERS)
    k = scaled(_heads(1, 3, n, "bhn", 12), eps)[0].transpose(0, 1).contiguous()  # [tokens, heads, d]
    table, start, lens, pages = batch([n], [0], 32)
    cos, sin = ref.tables(n, 64)
    w = torch.rand(ref.D, generator=torch.Generator().manual_seed(3)) + 0.5
    cache = empty_cache(mx, pages, 3, 32)
    want = ref.Cache(*cache)
    y, size = ref.turned(k.cpu(), w, eps, cos[:, None], sin[:, None], "halves")
    v = torch.ones_like(k)
    ref.append(want, y, v.cpu().double(), table, start, lens)
    mx.cache_append(k, v, *cache, table.cuda(), ints(start), ints(lens), w.cuda(), eps, cos.cuda(), sin.cuda(), None, "halves")
    check_append(cache, want, y, size)
    assert math.isfinite(float(ref.Cache(*cache).k.abs().max()))
