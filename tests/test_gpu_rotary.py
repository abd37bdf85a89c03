"""Rotary positions with several axes (fsx_rotary_rows) against the formula in 64 bits, on the CPU.

Tolerance, with u = 2^-24: the angle within its eighth of a turn is rounded three times (to fp32, the constant, the product), 3 u
relative, which moves a sine or cosine by at most 3 u x max(sin x, cos x) <= 1.7 u for x <= pi / 4; the polynomials end in one
rounding (u) and hold less than 0.6 u of roundings further in and 0.03 u of what they leave out: 3.4 u in all, and the fraction of
a turn adds 2^-32 turns (1.5e-9 = 0.03 u).  The product and the fma round once each.  So an output is off by at most
(4 u + 2 u) (|x_a| + |x_b|), and half a step of its type.  The reference's own angle, a product in 64 bits, is off by 2^-53 of it."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = 2.0 ** -24


def reference(x, positions, plan, inverse):
    """Output and tolerance without the output's rounding, [rows][heads][channels] in 64 bits."""
    n = len(plan.axis)
    angle = positions.to(F64)[torch.from_numpy(plan.axis).long()].t() * torch.from_numpy(plan.freq)
    c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if plan.layout == fsx.ROTARY_ADJACENT else (slice(0, n), slice(n, 2 * n))
    x = x.to(F64)
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    t = (6 * U + 2.0 ** -53 * angle.abs()[:, None]) * (x[..., a].abs() + x[..., b].abs())
    tol[..., a], tol[..., b] = t, t
    return y, tol


def check(got, x, positions, plan, inverse=False):
    y, tol = reference(x, positions, plan, inverse)
    tol = tol + torch.finfo(x.dtype).eps / 2 * (y.abs() + tol)
    n = 2 * len(plan.axis)
    got = got.cpu().to(F64)
    worst = ((got - y).abs() / (tol + 1e-300))[..., :n].max()
    assert bool(((got - y).abs() <= tol)[..., :n].all()), float(worst)
    assert torch.equal(got[..., n:], y[..., n:])


def inputs(rows, heads, dim, axes, dtype, far=100, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(rows, heads, dim, generator=g).to(dtype), torch.randint(-far, far + 1, (axes, rows), generator=g, dtype=torch.int32)


SECTIONS = [(128, (64,)), (128, (16, 24, 24)), (128, (22, 21, 21)), (64, (8, 12, 12)), (80, (20, 20)), (96, (16, 16, 15)), (72, (9, 9, 9, 9)),
            (256, (32, 48, 48)), (128, (8, 8, 16)), (2, (1,)), (7, (1, 0, 2)), (1024, (128,)), (12, (4,))]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", [fsx.ROTARY_HALVES, fsx.ROTARY_ADJACENT], ids=["halves", "adjacent"])
@pytest.mark.parametrize("dim,sections", SECTIONS, ids=str)
def test_sections(dim, sections, layout, dtype):
    for rows, heads, joint, inverse in ((1, 1, True, False), (5, 3, False, True), (33, 16, True, False)):
        plan = fsx.RotaryPlan.sections(sections, joint=joint, layout=layout)
        x, p = inputs(rows, heads, dim, len(sections), dtype, seed=rows)
        out = torch.full((rows, heads, dim), 7.0, dtype=dtype, device="cuda")
        fsx.rotary_rows(x.cuda(), out, p.cuda(), plan, inverse)
        check(out, x, p, plan, inverse)


@pytest.mark.parametrize("far", [0, 1, 16001, 1 << 20, 2 ** 31 - 1])
def test_far_positions_and_any_frequency(far):
    """Frequencies of 1 and more, none, negative ones, and the farthest positions, both ends among them."""
    plan = fsx.RotaryPlan([0] * 12, [1.0, 0.0, -0.75, math.pi, 2 * math.pi, 1e-9, 12345.678, -(2.0 ** 20), 2.0 ** 20, 0.1, 1e-300, 3.0])
    for dtype in (F32, BF16):
        x, p = inputs(64, 2, 24, 1, dtype, far=far, seed=3)
        p[0, 0], p[0, 1] = far, -far
        if far == 2 ** 31 - 1:
            p[0, 2] = -2 ** 31
        out = torch.empty_like(x, device="cuda")
        fsx.rotary_rows(x.cuda(), out, p.cuda(), plan)
        check(out, x, p, plan)


@pytest.mark.parametrize("rows,heads", [(1, 40), (16, 72), (2047, 3), (2048, 9), (6000, 40), (40000, 1)])
def test_many_rows(rows, heads):
    """Every way the rows and heads are shared out over workgroups."""
    plan = fsx.RotaryPlan.sections((16, 24, 24))
    x, p = inputs(rows, heads, 128, 3, BF16, seed=rows)
    out = torch.empty_like(x, device="cuda")
    fsx.rotary_rows(x.cuda(), out, p.cuda(), plan)
    check(out, x, p, plan)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("layout", [fsx.ROTARY_HALVES, fsx.ROTARY_ADJACENT], ids=["halves", "adjacent"])
def test_in_place_and_strided(layout, dtype):
    """Queries and keys of a projection's rows in place, the values beside them untouched; odd strides; positions [rows][axes]."""
    plan = fsx.RotaryPlan.sections((8, 12, 8), layout=layout)  # the last 8 channels stay
    for gap in (0, 8, 5):
        x, p = inputs(37, 14, 64 + gap, 3, dtype, seed=gap)
        dev, pd = x.cuda(), p.t().contiguous().cuda().t()
        qk = dev[:, 1:11, gap:]
        fsx.rotary_rows(qk, qk, pd, plan)
        check(dev[:, 1:11, gap:], x[:, 1:11, gap:], p, plan)
        rest = dev.cpu().clone()
        rest[:, 1:11, gap:] = x[:, 1:11, gap:]
        assert torch.equal(rest, x)
        # beside the source, in the same rows
        dev = x.cuda()
        fsx.rotary_rows(dev[:, :5, gap:], dev[:, 7:12, gap:], pd, plan)
        check(dev[:, 7:12, gap:], x[:, :5, gap:], p, plan)
        assert torch.equal(dev[:, :7].cpu(), x[:, :7]) and torch.equal(dev[:, 12:].cpu(), x[:, 12:])
        # heads before rows
        y = torch.empty(14, 37, 64, dtype=dtype, device="cuda").transpose(0, 1)
        fsx.rotary_rows(x.cuda()[..., gap:], y, pd, plan)
        check(y, x[..., gap:], p, plan)


def test_gradient():
    """The rotation back is the gradient: against the formula's own by autograd in 64 bits, and against differences."""
    plan = fsx.RotaryPlan.sections((5, 7), joint=False, layout=fsx.ROTARY_ADJACENT)
    x, p = inputs(19, 3, 26, 2, F32, seed=4)
    dy = torch.randn(19, 3, 26, generator=torch.Generator().manual_seed(5))
    dx = torch.empty_like(dy, device="cuda")
    fsx.rotary_rows(dy.cuda(), dx, p.cuda(), plan, inverse=True)
    leaf = x.to(F64).requires_grad_()
    n = 12
    angle = p.to(F64)[torch.from_numpy(plan.axis).long()].t() * torch.from_numpy(plan.freq)
    a, b = leaf[..., 0:2 * n:2], leaf[..., 1:2 * n:2]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    y = torch.cat([torch.stack([a * c - b * s, b * c + a * s], 3).flatten(2), leaf[..., 2 * n:]], 2)
    (y * dy.to(F64)).sum().backward()
    t = 6 * U * (dy[..., 0:2 * n:2].abs() + dy[..., 1:2 * n:2].abs()).to(F64)
    err = (dx.cpu().to(F64) - leaf.grad).abs()
    assert bool((err[..., 0:2 * n:2] <= t + U * 8).all()) and bool((err[..., 1:2 * n:2] <= t + U * 8).all())
    # a step of x in one direction: the rotation is linear, so the difference is exact but for the roundings of both outputs
    d = torch.randn(19, 3, 26, generator=torch.Generator().manual_seed(6))
    out = [torch.empty_like(dy, device="cuda") for _ in "ab"]
    for o, z in zip(out, (x + d, x)):
        fsx.rotary_rows(z.cuda(), o, p.cuda(), plan)
    step = (x + d).to(F64) - x.to(F64)
    left = ((out[0] - out[1]).cpu().to(F64) * dy.to(F64)).sum()
    right = (dx.cpu().to(F64) * step).sum()

    def pairs(z):  # |x_a| + |x_b| in both places
        z = z.abs().to(F64)
        z[..., 0:2 * n:2] = z[..., 1:2 * n:2] = z[..., 0:2 * n:2] + z[..., 1:2 * n:2]
        return z

    # an output is off by 6 u of its pair and its rounding, the difference of two rounds once more
    bound = 8 * U * ((pairs(x + d) + pairs(x)) * dy.abs().to(F64)).sum() + 7 * U * (pairs(dy) * step.abs()).sum()
    assert abs(float(left - right)) <= float(bound)


def test_infinities_and_nan_stay_in_their_pair():
    plan = fsx.RotaryPlan.sections((32,))
    x, p = inputs(3, 2, 64, 1, BF16, seed=1)
    x[1, 1, 5], x[2, 0, 40] = math.inf, math.nan
    out = torch.empty_like(x, device="cuda")
    fsx.rotary_rows(x.cuda(), out, p.cuda(), plan)
    bad = ~torch.isfinite(out.cpu())
    assert bad.nonzero().tolist() == [[1, 1, 5], [1, 1, 37], [2, 0, 8], [2, 0, 40]]


def test_captured_and_on_another_stream():
    plan = fsx.RotaryPlan.sections((16, 24, 24))
    x, p = inputs(50, 6, 128, 3, BF16, seed=8)
    xd, pd, out = x.cuda(), p.cuda(), torch.zeros(50, 6, 128, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fsx.rotary_rows(xd, out, pd, plan, stream=side)
    side.synchronize()
    check(out, x, p, plan)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fsx.rotary_rows(xd, out, pd, plan)
    for seed in (1, 2, 3):
        x, p = inputs(50, 6, 128, 3, BF16, seed=seed)
        xd.copy_(x)
        pd.copy_(p)
        graph.replay()
        torch.cuda.synchronize()
        check(out, x, p, plan)
        eager = torch.empty_like(out)
        fsx.rotary_rows(xd, eager, pd, plan)
        assert torch.equal(eager, out)


def test_rows_past_32_bits():
    """The last rows of a tensor of more than 2^31 elements."""
    rows, heads, dim = 20000, 512, 256  # 2.6e9 elements
    plan = fsx.RotaryPlan.sections((128,))
    x = torch.empty(rows, heads, dim, dtype=BF16, device="cuda")
    out = torch.empty_like(x)
    tail, _ = inputs(2, heads, dim, 1, BF16, seed=2)
    x[-2:] = tail.cuda()
    p = torch.arange(rows, dtype=torch.int32, device="cuda")[None]
    fsx.rotary_rows(x, out, p, plan)
    check(out[-2:], tail, p[:, -2:].cpu(), plan)


def test_host_tensors_are_refused():
    plan = fsx.RotaryPlan.sections((32,))
    x, p = inputs(3, 2, 64, 1, BF16)
    for a, b, c in ((x, x.cuda(), p.cuda()), (x.cuda(), x, p.cuda()), (x.cuda(), x.cuda(), p)):
        with pytest.raises(ValueError, match="current device"):
            fsx.rotary_rows(a, b, c, plan)
    with pytest.raises(ValueError, match="int32"):
        fsx.rotary_rows(x.cuda(), x.cuda(), p.cuda().float(), plan)
    with pytest.raises(fsx.FsxError, match="axis"):
        fsx.rotary_rows(x.cuda(), x.cuda(), p.cuda(), fsx.RotaryPlan([1] * 32, [1.0] * 32))
