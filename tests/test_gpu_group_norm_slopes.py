"""Derivatives of the activations in the fp32 backward pass, over the whole range of t.

With mean 0, rstd 1, no w and b, t is x; with dz 1 at one voxel and 0 elsewhere, db is the derivative at that voxel's t.
Tolerances, u = 2^-24.  SiLU: an exponential 7 u (the instruction's 4, its argument's and its factor's rounding), 1 + e^-t one, a reciprocal 2, so sigmoid s
10 u and y = t s 11 u: s + y - y s is within 24 u (s + |y| + |y s|).  GELU, normal distribution P, density p: e^(-t^2 / 2) is off by the instruction's 4 u
and half of t^2 times the argument's 2.3 u (two products and the constant), the polynomial by 8 u (3.4e-7 in fp32 arithmetic, and the reciprocal), the
product, the sum and 1 - P by one each: P + t p is within (16 + 1.25 t^2) u (P + |t| p).  Below 2^-126 the instructions flush to 0."""
import math

import numpy as np
import pytest
import torch

from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("name,reach", [("silu", 85.0), ("gelu", 13.0)])
@pytest.mark.parametrize("voxels", [1, 40000])
@pytest.mark.parametrize("zt", [torch.float32, torch.bfloat16])
def test_slopes_keep_their_digits(name, reach, voxels, zt):
    c = 2048
    t = np.linspace(-reach, reach, c)
    t[1::2] = np.random.default_rng(0).uniform(-reach / 4, reach / 4, c // 2)
    t = t.astype(np.float32)
    x = torch.zeros(1, 1, 1, voxels, c, device="cuda")
    dz = torch.zeros(x.shape, dtype=zt, device="cuda")
    x[0, 0, 0, voxels // 2], dz[0, 0, 0, voxels // 2] = torch.from_numpy(t).cuda(), 1.0
    mr = torch.tensor([0.0, 1.0], device="cuda").repeat(1, c // 8, 1).contiguous()
    p = B.group_norm(c // 8, None, None, name)
    ws = torch.empty(B.lamp_group_norm_workspace_bytes(p, x), dtype=torch.uint8, device="cuda")
    dx, db = torch.empty_like(x), torch.empty(c, device="cuda")
    B.lamp_group_norm_act_bwd(p, dz, x, mr, dx, None, db, ws)
    v = t.astype(np.float64)
    if name == "silu":                                                    # 1 - s as it is, not from s: no digit cancels at either end
        s, r = 1 / (1 + np.exp(-v)), 1 / (1 + np.exp(v))
        ref, e = s + v * s * r, 24 * U * (s + np.abs(v) * s + np.abs(v) * s * s)
    else:
        below, density = np.array([0.5 * math.erfc(-a / math.sqrt(2)) for a in v]), np.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        ref, e = below + v * density, (16 + 1.25 * v * v) * U * (below + np.abs(v) * density)
    bad = np.abs(db.double().cpu().numpy() - ref) > e + 2.0 ** -126
    assert not bad.any(), (bad.sum(), t[bad][:6], db.cpu().numpy()[bad][:6], ref[bad][:6])
    if voxels == 1:                                                       # the pass that applies: dx = dt - its group's mean - t mean(dt t)
        g = ref.reshape(-1, 8)
        want = (g - g.mean(1, keepdims=True) - v.reshape(-1, 8) * (g * v.reshape(-1, 8)).mean(1, keepdims=True)).reshape(-1)
        a, m = np.abs(v.reshape(-1, 8)), e.reshape(-1, 8) + 8 * U * np.abs(g)
        tol = (m + m.mean(1, keepdims=True) + a * (m * a).mean(1, keepdims=True)).reshape(-1) + 2.0 ** -120
        assert (np.abs(dx.view(-1).double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("name", ["silu", "gelu"])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_slopes_far_out(name, dt):
    """0 below and 1 above, however far t is."""
    t = torch.tensor([-3e38, -1e30, -1e10, -1e3, 1e3, 1e10, 1e30, 3e38], device="cuda")
    x = t.to(dt).view(1, 1, 1, 1, 8)
    mr = torch.tensor([0.0, 1.0], device="cuda").repeat(1, 8, 1).contiguous()
    p = B.group_norm(8, None, None, name)
    ws = torch.empty(B.lamp_group_norm_workspace_bytes(p, x), dtype=torch.uint8, device="cuda")
    db = torch.empty(8, device="cuda")
    B.lamp_group_norm_act_bwd(p, torch.ones_like(x), x, mr, torch.empty_like(x), None, db, ws)
    assert (db == torch.tensor([0.0] * 4 + [1.0] * 4, device="cuda")).all(), db
