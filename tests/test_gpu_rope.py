"""Norm and rotation of heads against the formula in 64 bits.

Tolerance: the result is rounded once to bf16 (2^-8 of it).  Before that, in
fp32 (2^-24 each): the sum of squares (8 fused steps, 4 of the tree: 12, halved
by the root), mean, eps, root, reciprocal and two products (6), the rotation's
two products and one sum (3): under 2^-19 of |a| + |b|, the normed pair."""
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


def _heads(B, H, N, order, seed):
    """bf16 [B, H, N, d] on the device, its axes in memory in this order."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, H, N, ref.D), generator=g) * torch.exp(torch.randn((H, 1, ref.D), generator=g))
    x = x.to(torch.bfloat16)
    at = ["bhn".index(a) for a in order]
    return x.permute(*at, 3).contiguous().permute(*[at.index(i) for i in range(3)], 3).cuda()


def _check(out, x, w, eps, cos, sin, pos, pairs):
    c = s = None
    if cos is not None:
        at = pos.long().cpu()
        c, s = cos.cpu()[at][:, None], sin.cpu()[at][:, None]
    y, size = ref.turned(x.cpu(), w.cpu() if w is not None else None, eps, c, s, pairs)
    err = (out.cpu().double() - y).abs()
    worst = float((err / (2.0 ** -8 * y.abs() + 2.0 ** -19 * size + 1e-38)).max())
    assert worst <= 1.0, worst


CASES = [
    # B, Hq, Hkv, N, rot, pairs, order, norm, gather
    (1, 1, 1, 1, 128, "interleaved", "bhn", True, False),
    (1, 1, 1, 1, 128, "halves", "bnh", True, True),
    (3, 5, 1, 17, 64, "halves", "bnh", True, True),
    (2, 8, 2, 33, 96, "interleaved", "nbh", True, True),
    (2, 40, 40, 15, 128, "interleaved", "bnh", False, False),
    (1, 24, 24, 130, 16, "halves", "bnh", True, False),
    (4, 3, 2, 7, 112, "halves", "hbn", False, True),
    (33, 32, 8, 1, 128, "halves", "bnh", True, True),
    (2, 6, 3, 100, 0, "halves", "bnh", True, False),
    (1, 40, 40, 2053, 128, "interleaved", "bnh", True, False),
    (1, 7, 1, 4097, 48, "halves", "bnh", True, True),
]


@pytest.mark.parametrize("case", CASES)
def test_against_64_bits(mx, case):
    B, Hq, Hkv, N, rot, pairs, order, norm, gather = case
    print(f"[rope] {case}", flush=True)
    q, k = _heads(B, Hq, N, order, 1), _heads(B, Hkv, N, order, 2)
    rows = 2 * N + 5
    cos, sin = (t.cuda() for t in ref.tables(rows, rot)) if rot else (None, None)
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(rows, (B, N), generator=g, dtype=torch.int32).cuda() if gather else None
    w = [(torch.rand(ref.D, generator=g) + 0.5).cuda() if norm else None for _ in range(2)]
    eps = 1e-6
    qo, ko = mx.qk_norm_rope(q, k, w[0], w[1], eps, cos, sin, pos, pairs)
    at = pos if gather else torch.arange(N).expand(B, N)
    _check(qo, q, w[0], eps, cos, sin, at, pairs)
    _check(ko, k, w[1], eps, cos, sin, at, pairs)
    assert qo.is_contiguous() and ko.is_contiguous()


def test_parts_of_one_projection_and_given_outputs(mx):
    """Views of a fused projection in, outputs with strides of their own; what lies between their rows stays."""
    B, N, Hq, Hkv = 2, 19, 4, 2
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn((B, N, Hq + 2 * Hkv, ref.D), generator=g).to(torch.bfloat16).cuda()
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    cos, sin = (t.cuda() for t in ref.tables(N, 128))
    buf = torch.full((B, N, Hq + 1, ref.D), 7.0, dtype=torch.bfloat16, device="cuda")
    kb = torch.full((Hkv, B, N, ref.D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, ko = buf[:, :, :Hq].transpose(1, 2), kb[..., :ref.D].transpose(0, 1)
    ones = torch.ones(ref.D, device="cuda")
    mx.qk_norm_rope(q, k, ones, None, 1e-5, cos, sin, None, "halves", qo, ko)
    at = torch.arange(N).expand(B, N)
    _check(qo, q, ones, 1e-5, cos, sin, at, "halves")
    _check(ko, k, None, 0.0, cos, sin, at, "halves")
    assert bool((buf[:, :, Hq] == 7).all()) and bool((kb[..., ref.D:] == 7).all())
    # a batch that is one tensor broadcast, and Q alone
    e = q[:1].expand(3, Hq, N, ref.D)
    eo, none = mx.qk_norm_rope(e, None, ones, None, 1e-5, cos, sin, None, "halves")
    assert none is None and torch.equal(eo[2], qo[0]) and torch.equal(eo[0], qo[0])


@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
def test_zeros_infinities_and_positions_outside_the_table(mx, pairs):
    B, H, N = 1, 2, 6
    q = _heads(B, H, N, "bhn", 9)
    q[0, 0, 0] = 0
    q[0, 0, 1, 5] = float("inf")
    q[0, 0, 2, 64] = float("nan")
    cos, sin = (t.cuda() for t in ref.tables(4, 64))
    pos = torch.tensor([[0, 1, 2, 3, 4, -1]], dtype=torch.int32, device="cuda")
    w = torch.ones(ref.D, device="cuda")
    o, _ = mx.qk_norm_rope(q, None, w, None, 1e-6, cos, sin, pos, pairs)
    assert bool((o[0, 0, 0] == 0).all())
    assert bool(o[0, 0, 2].isnan().all())                  # its sum of squares is NaN
    assert bool(o[0, 0, 1, 5].isnan())                     # inf * (1 / inf)
    for n in (4, 5):                                        # no such position: the rotated channels only
        assert bool(o[0, :, n, :64].isnan().all()) and bool(o[0, :, n, 64:].isfinite().all())
    _check(o[:, 1:, :4], q[:, 1:, :4], w, 1e-6, cos, sin, pos[:, :4], pairs)


def test_large_and_small_magnitudes(mx):
    """Rows whose squares leave no digits to eps, and rows that eps carries."""
    q = _heads(1, 3, 8, "bhn", 11)
    q[0, 0] *= 2.0 ** 40
    q[0, 1] *= 2.0 ** -40
    w = torch.ones(ref.D, device="cuda")
    o, _ = mx.qk_norm_rope(q, None, w, None, 1e-6)
    _check(o, q, w, 1e-6, None, None, None, "halves")
