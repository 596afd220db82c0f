"""Rotary embedding with several axes on the GPU against the fp64 oracle."""
import numpy as np
import pytest

from oracle import paged
from paged_util import BF16_HALF_STEP, bf16

pytestmark = pytest.mark.gpu


def sections(axes, half):
    return [i * axes // half for i in range(half)]


def interleaved(axes, half):
    return [i % axes for i in range(half)]


def tolerance(x, want, f32):
    # fp32: the table's value half a step off (2^-24), two products and a sum rounded: at most 4 * 2^-24 of |lo| + |hi| <= 2 max |x|
    fp32 = 8 * 2.0 ** -24 * np.abs(x).max(axis=-1, keepdims=True, initial=0.0)
    return fp32 + (0.0 if f32 else BF16_HALF_STEP * np.abs(want))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("T,hq,hkv,d,axes,layout,fused", [
    (1, 1, 1, 8, 1, sections, False), (17, 3, 1, 64, 3, sections, True), (130, 8, 2, 128, 3, interleaved, True),
    (65, 5, 5, 104, 2, interleaved, False), (7, 24, 24, 128, 4, sections, False), (5000, 2, 1, 40, 3, sections, False),
    (33, 130, 1, 16, 2, sections, False), (300, 4, 0, 96, 3, sections, False)])
def test_against_the_oracle(T, hq, hkv, d, axes, layout, fused, inverse, f32):
    import torch
    import paper_2504_20490_amd as A
    rng = np.random.default_rng(T + d)
    dtype = torch.float32 if f32 else torch.bfloat16
    x = rng.standard_normal((T, hq + hkv, d))
    x = x.astype(np.float32).astype(np.float64) if f32 else bf16(x)
    dev = torch.from_numpy(x).to(dtype).cuda()
    q, k = dev[:, :hq], dev[:, hq:] if hkv else None
    if not fused:
        q, k = q.contiguous(), k.contiguous() if hkv else None
    n = 4000
    table = torch.empty(n, d // 2, 2, device="cuda")
    A.rope_table(table, n, d)
    positions = rng.integers(0, n, (axes, T))
    pair_axis = layout(axes, d // 2)
    rope = A.RopeAxes(table, n, torch.from_numpy(positions).int().cuda(), pair_axis)
    q_out = torch.full((T, hq, d), float("nan"), dtype=dtype, device="cuda")
    k_out = torch.full((T, hkv, d), float("nan"), dtype=dtype, device="cuda") if hkv else None
    A.rope_axes_qk(rope, q, k, q_out, k_out, inverse=inverse)
    torch.cuda.synchronize()
    want = paged.turn_axes(x, positions, pair_axis, inverse=inverse)
    for got, ref, src in ((q_out, want[:, :hq], x[:, :hq]), (k_out, want[:, hq:], x[:, hq:])):
        if got is not None:
            assert (np.abs(got.double().cpu().numpy() - ref) <= tolerance(src, ref, f32)).all()
    # in place, the same bits
    q2, k2 = q.clone(), None if k is None else k.clone()
    A.rope_axes_qk(rope, q2, k2, q2, k2, inverse=inverse)
    torch.cuda.synchronize()
    assert torch.equal(q2, q_out) and (k is None or torch.equal(k2, k_out))


def test_one_axis_equals_the_plan_rotation():
    import torch
    import paper_2504_20490_amd as A
    lengths, hq, hkv, d = [17, 64, 111], 4, 2, 128
    cu, _, T = A.build_cu_seqlens(lengths)
    x = torch.randn(T, hq + hkv, d, device="cuda").bfloat16()
    table = torch.empty(111, d // 2, 2, device="cuda")
    A.rope_table(table, 111, d)
    a = [torch.empty(T, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hq, hkv)]
    A.rope_qk(A.Plan(cu, hq, hkv, d), x[:, :hq], x[:, hq:], a[0], a[1], table, 111)
    pos = torch.cat([torch.arange(n) for n in lengths]).int().cuda()
    A.rope_axes_qk(A.RopeAxes(table, 111, pos), x[:, :hq], x[:, hq:], a[2], a[3])
    torch.cuda.synchronize()
    for y, z in ((a[0], a[2]), (a[1], a[3])):       # (one may contract a product and a sum: a rounding of bf16 at most)
        assert ((y.float() - z.float()).abs() <= 2.0 ** -7 * y.float().abs() + 2.0 ** -20).all()


def test_positions_outside_the_table():
    """The pairs of the axis are NaN for that token, everything else is right."""
    import torch
    import paper_2504_20490_amd as A
    d, n = 64, 50
    table = torch.empty(n, d // 2, 2, device="cuda")
    A.rope_table(table, n, d)
    positions = torch.tensor([[0, 49, 3, 50], [1, -1, 1 << 30, 4]], dtype=torch.int32, device="cuda")
    pair_axis = sections(2, d // 2)
    x = torch.randn(4, 3, d, device="cuda")
    out = torch.empty_like(x)
    A.rope_axes_qk(A.RopeAxes(table, n, positions, pair_axis), x, None, out, None)
    torch.cuda.synchronize()
    want = paged.turn_axes(x.double().cpu().numpy(), positions.cpu().numpy().clip(0, n - 1), pair_axis)
    got = out.double().cpu().numpy()
    bad = np.zeros((4, 3, d), dtype=bool)
    for t, axis in ((1, 1), (2, 1), (3, 0)):
        cols = [i for i in range(d // 2) if pair_axis[i] == axis]
        bad[t][:, cols + [c + d // 2 for c in cols]] = True
    assert np.array_equal(np.isnan(got), bad)
    assert (np.abs(got - want)[~bad] <= 8 * 2.0 ** -24 * float(x.abs().max())).all()


@pytest.mark.parametrize("f32", [False, True])
def test_the_inverse_is_the_gradient(f32):
    """f(x) = sum(w * rope(x)): its gradient by the inverse rotation of w, against the formula's (the transposed map) and differences of
    the oracle's forward in 64 bits."""
    import torch
    import paper_2504_20490_amd as A
    T, h, d, axes = 5, 2, 16, 3
    rng = np.random.default_rng(0)
    pair_axis, positions = interleaved(axes, d // 2), rng.integers(0, 30, (axes, T))
    w = bf16(rng.standard_normal((T, h, d)))
    table = torch.empty(30, d // 2, 2, device="cuda")
    A.rope_table(table, 30, d)
    rope = A.RopeAxes(table, 30, torch.from_numpy(positions).int().cuda(), pair_axis)
    dw = torch.from_numpy(w).to(torch.float32 if f32 else torch.bfloat16).cuda()
    grad = torch.empty_like(dw)
    A.rope_axes_qk(rope, dw, None, grad, None, inverse=True)
    torch.cuda.synchronize()
    got = grad.double().cpu().numpy()
    x = rng.standard_normal((T, h, d))
    f = lambda y: float((w * paged.turn_axes(y, positions, pair_axis)).sum())
    for _ in range(20):
        at = tuple(int(rng.integers(n)) for n in (T, h, d))
        e = np.zeros_like(x)
        e[at] = 0.5                                    # (the map is linear: any step is exact but for rounding)
        diff = f(x + e) - f(x - e)
        assert abs(got[at] - diff) <= 1e-9 + float(tolerance(w, np.array(diff), f32).max())


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("d", range(8, 129, 8))
def test_every_head_dim(d, f32):
    test_against_the_oracle(37, 5, 2, d, 3, interleaved, True, d % 16 == 0, f32)
