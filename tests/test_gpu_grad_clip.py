"""Gradient norm, clipping and the scaled update on the GPU against fp64.

Tolerances.  Squares are added in fp32 over 8 neighbours (8 roundings, 2^-24 relative each, on non-negative terms), in fp64 beyond; the
norm is the square root of the sum, so half of that relative error, and one rounding to fp32: |norm - ref| <= 5 * 2^-24 ref.  factor: one
division more, |factor - ref| <= 6 * 2^-24 ref.  A clipped value: one product more, 7 * 2^-24 relative, and half a step of its type
(bf16 2^-8; below the normal range half of the smallest step)."""
import math

import numpy as np
import pytest
import torch

from oracle import group as G
from oracle import optim
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def scratch(lst):
    return torch.full((B.lamp_grad_norm_workspace_bytes(lst),), 0xFF, dtype=torch.uint8, device="cuda")


def scalars():
    return torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")


def host(t):
    return t.double().cpu().numpy()


def check_clip(grads, max_norm, outs=None):
    src = [host(g) for g in grads]
    lst = B.grad_list(grads, outs)
    norm, factor = scalars()
    B.lamp_grad_clip(lst, max_norm, norm, factor, scratch(lst))
    rn, rf, ro = G.clip(src, max_norm)
    assert abs(norm.item() - rn) <= 5 * U * rn, (norm.item(), rn)
    # near the border the rounded norm decides
    if abs(rn - max_norm) > 10 * U * rn:
        assert abs(factor.item() - rf) <= 6 * U * rf, (factor.item(), rf)
    f = factor.item()
    for t, s in zip(grads if outs is None else outs, src):
        half = 2.0 ** -8 if t.dtype is torch.bfloat16 else U
        tiny = 2.0 ** -134 if t.dtype is torch.bfloat16 else 2.0 ** -150
        assert (np.abs(host(t) - s * f) <= (half + 2 * U) * np.abs(s * f) + tiny).all()
    return norm, factor


SIZES = [[1], [3], [8], [7, 1, 9], [256, 100000], [8192, 8191, 8193, 16384], [5] * 130, [1000] * 119 + [7] * 3, [3] * 2100, [2500000, 0, 33]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("ratio", [0.3, 2.0])
def test_clip_matches_fp64(sizes, kind, ratio):
    g = torch.Generator(device="cuda").manual_seed(len(sizes))
    grads = []
    for i, n in enumerate(sizes):
        dt = torch.bfloat16 if kind == "bf16" or (kind == "mixed" and i % 2) else torch.float32
        off = i % 5                                                   # views at every alignment
        grads.append((torch.randn(n + off, device="cuda", generator=g) * 0.01).to(dt)[off:])
    total = math.sqrt(sum(float((host(t) ** 2).sum()) for t in grads))
    before = [t.clone() for t in grads]
    _, factor = check_clip(grads, total * ratio)
    if ratio > 1:
        assert factor.item() == 1.0 and all(torch.equal(a, b) for a, b in zip(grads, before))


@pytest.mark.parametrize("shift", [0, 1, 3])
def test_outputs_elsewhere_and_at_another_alignment(shift):
    grads = [torch.randn(n, device="cuda").to(dt) for n, dt in ((70001, torch.float32), (33000, torch.bfloat16), (9, torch.float32))]
    room = [torch.full((t.numel() + 8,), 5.0, dtype=t.dtype, device="cuda") for t in grads]
    outs = [r[shift:shift + t.numel()] for r, t in zip(room, grads)]
    before = [t.clone() for t in grads]
    check_clip(grads, 10.0, outs)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    for r, t in zip(room, grads):
        assert (r[:shift] == 5).all() and (r[shift + t.numel():] == 5).all()
    check_clip(grads, 1e6, outs)                                       # factor 1: copied


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e18, 1e30])
def test_squares_outside_of_fp32(scale):
    grads = [torch.randn(5000, device="cuda") * scale, torch.zeros(300, device="cuda"), torch.randn(3, device="cuda") * scale]
    grads[0][::3] *= 1e-8                                              # small beside large, and alone in their eight
    grads[0][64:128] = 1e-8 * scale
    check_clip(grads, 0.5 * scale)


def test_not_finite():
    for bad, want_norm, want_factor in ((float("inf"), math.inf, 0.0), (float("nan"), math.nan, math.nan)):
        for at in (0, 4999):
            t = torch.ones(5000, device="cuda")
            t[at] = bad
            lst = B.grad_list([t])
            norm, factor = scalars()
            B.lamp_grad_norm(lst, 1.0, norm, factor, scratch(lst))
            assert np.array_equal([norm.item(), factor.item()], [want_norm, want_factor], equal_nan=True)
            B.lamp_grad_clip(lst, 1.0, norm, factor, scratch(lst))
            assert t[at].isnan() and (t[1] == 0 if want_factor == 0 else t[1].isnan())
    big = torch.full((4,), 3e38, device="cuda")
    lst = B.grad_list([big])
    norm, factor = scalars()
    B.lamp_grad_norm(lst, 1.0, norm, factor, scratch(lst))
    assert norm.item() == math.inf and factor.item() == 0.0            # 6e38 is no fp32 number


def test_nothing_and_zero():
    for lst in (B.grad_list([]), B.grad_list([torch.empty(0, device="cuda")]), B.grad_list([torch.zeros(100, device="cuda")])):
        for f in (B.lamp_grad_norm, B.lamp_grad_clip):
            norm, factor = scalars()
            f(lst, 0.0, norm, factor, torch.empty(65536, dtype=torch.uint8, device="cuda"))
            assert norm.item() == 0.0 and factor.item() == 1.0


def test_norm_alone_leaves_the_gradients():
    t = torch.randn(100001, device="cuda")
    c = t.clone()
    lst = B.grad_list([t])
    norm, factor = scalars()
    B.lamp_grad_norm(lst, 1.0, norm, None, scratch(lst))
    assert torch.equal(t, c) and abs(norm.item() - float(c.double().norm())) <= 5 * U * norm.item()
    B.lamp_grad_norm(lst, math.inf, norm, factor, scratch(lst))
    assert factor.item() == 1.0


def test_repeats_bit_for_bit_and_in_graphs_that_share_scratch():
    grads = [torch.randn(n, device="cuda") for n in (300000, 17, 5000)]
    outs = [torch.empty_like(t) for t in grads]
    lst = B.grad_list(grads, outs)
    ws = scratch(lst)
    norm, factor = scalars()
    B.lamp_grad_clip(lst, 1.0, norm, factor, ws)
    first = [norm.item(), factor.item()] + [t.clone() for t in outs]
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.lamp_grad_clip(lst, 1.0, norm, factor, ws)
    for g in graphs * 3:
        for t in outs:
            t.zero_()
        g.replay()
        assert norm.item() == first[0] and factor.item() == first[1] and all(torch.equal(a, b) for a, b in zip(outs, first[2:]))
    grads[0].mul_(2.0)
    graphs[0].replay()
    assert abs(norm.item() - math.sqrt(sum(float(t.double().square().sum()) for t in grads))) <= 5 * U * norm.item()


@pytest.mark.parametrize("n", [1, 7, 4096, 100003])
def test_scaled_update_is_the_update_of_scaled_gradients(n):
    r = np.random.default_rng(n)
    g, w, v = (r.standard_normal(n).astype(np.float32) for _ in range(3))
    v = np.abs(v)
    s = np.float32(0.37)
    dev = [torch.from_numpy(a.copy()).cuda() for a in (g, w, v)]
    plain = [t.clone() for t in dev]
    p16, q16 = torch.empty(n, dtype=torch.bfloat16, device="cuda"), torch.empty(n, dtype=torch.bfloat16, device="cuda")
    B.lamp_rmsprop_step_scaled(dev[0], torch.full((1,), float(s), device="cuda"), dev[1], dev[2], p16, 1e-2, 0.9, 1e-6)
    B.lamp_rmsprop_step((plain[0] * torch.tensor(float(s), device="cuda")), plain[1], plain[2], q16, 1e-2, 0.9, 1e-6)
    assert torch.equal(dev[1], plain[1]) and torch.equal(dev[2], plain[2]) and torch.equal(p16, q16)
    rw, rv = optim.rmsprop_step(w, g.astype(np.float64) * float(s), v, 1e-2, 0.9, 1e-6)[:2]
    assert np.abs(host(dev[1]) - rw).max() < 1e-5 and np.abs(host(dev[2]) - rv).max() < 1e-5


def test_list_refuses_overlaps_and_foreign_tensors():
    a, b = torch.zeros(100, device="cuda"), torch.zeros(100, device="cuda")
    for tensors, outs in (([a, a], None), ([a, a[50:]], None), ([a[:60], a[50:]], None), ([a, b], [b, torch.zeros_like(b)]), ([a[:50], b[:50]], [a[25:75], b[50:]]),
                          ([a, b], [torch.zeros_like(a), a])):
        with pytest.raises(ValueError):
            B.grad_list(tensors, outs)
    assert B.grad_list([a[:50], a[50:]]).count == 2                      # neighbours
    assert B.grad_list([a, a], [torch.zeros_like(a), torch.zeros_like(a)]).count == 2
    for bad, outs in (([a.half()], None), ([a.cpu()], None), ([torch.zeros(10, 10, device="cuda")[:, ::2]], None), ([a], [b[:50]]), ([a], [b.bfloat16()])):
        with pytest.raises(ValueError):
            B.grad_list(bad, outs)
    lst = B.grad_list([a])
    n, f = scalars()
    with pytest.raises(B.LampError):
        B.lamp_grad_norm(lst, 1.0, n, f, None)
    with pytest.raises(ValueError):
        B.lamp_grad_norm(lst, 1.0, n.double(), f, scratch(lst))
