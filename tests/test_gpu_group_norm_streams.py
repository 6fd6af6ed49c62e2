"""The streaming form of the group norm where the other tests do not take it: gradients of w and b over many samples, tensors that are applied in
short runs (64 units per thread of a resident grid and more), given sums of tensors with many groups or many channels per group.

Tolerances as in the operator's other tests (derived there); the large shapes are compared with fp64 on the GPU, a sample at a time."""

import pytest
import torch

from paper_2006_12575_b200 import binding as B
from test_gpu_group_norm import TYPES, case, check_backward, check_forward, dev, host, scratch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shape", [(6, (26, 26, 26), 24, 3), (40, (20, 20, 20), 32, 4), (640, (1, 5, 9), 64, 8), (70000, (1, 1, 2), 8, 2)], ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_many_samples(shape, types):
    n, dhw, c, groups = shape
    xt, zt = TYPES[types]
    r, x, w, b = case(shape, 1)
    tx, tg = dev(x, xt), dev(r.standard_normal(x.shape), zt)
    p = B.group_norm(groups, dev(w), dev(b), "silu")
    ws, z, mr = scratch(p, tx), torch.empty(x.shape, dtype=zt, device="cuda"), torch.empty(n, groups, 2, device="cuda")
    B.lamp_group_norm_act_fwd(p, tx, z, mr, ws)
    check_forward(z, mr, host(tx), w, b, shape, "silu", 0.0, 1e-5, zt)
    for dw, db in ((True, True), (True, False), (False, True)):
        dw, db = (torch.full((c,), float("nan"), device="cuda") if k else None for k in (dw, db))
        dx = torch.full_like(tx, float("nan"))
        B.lamp_group_norm_act_bwd(p, tg, tx, mr, dx, dw, db, ws)
        check_backward(dx, dw, db, host(tg), host(tx), host(mr), w, b, shape, "silu", 0.0, 1e-5, xt)


def sample_reference(x, dz, mean, rstd, w, b, groups, name):
    """fp64 of one sample [v, c] on the GPU: z, dx, dw, db, and the magnitudes that the tolerances take."""
    v, c = x.shape
    m, s = (a.repeat_interleave(c // groups) for a in (mean, rstd))
    xh = (x - m) * s
    t = xh * w + b
    if name == "silu":
        sig = torch.sigmoid(t)
        z, slope = t * sig, sig * (1 + t * torch.sigmoid(-t))
    else:
        z, slope = torch.where(t > 0, t, 0.1 * t), torch.where(t > 0, 1.0, 0.1).double()
    dt = dz * slope
    per = lambda a: a.view(v, groups, -1).mean((0, 2)).repeat_interleave(c // groups)                      # noqa: E731
    level, along = per(w * dt), per(w * dt * xh)
    return z, t, xh, dt, (w * dt - level - xh * along) * s, s


@pytest.mark.parametrize("shape", [(3, 13000, 2048, 32), (200, 4200, 64, 8)], ids=str)
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("name", ["silu", "leaky_relu"])
def test_short_runs(shape, types, name):
    n, v, c, groups = shape
    xt, zt = TYPES[types]
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dz = torch.empty(n, 1, 1, v, c, dtype=xt, device="cuda"), torch.empty(n, 1, 1, v, c, dtype=zt, device="cuda")
    for i in range(n):
        x[i], dz[i] = torch.randn(1, 1, v, c, device="cuda", generator=g) * 1.5 + 0.3, torch.randn(1, 1, v, c, device="cuda", generator=g)
    w, b = 1 + 0.3 * torch.randn(c, device="cuda", generator=g), 0.2 * torch.randn(c, device="cuda", generator=g)
    p = B.group_norm(groups, w, b, name, 0.1)
    ws, z, dx = scratch(p, x), torch.full_like(dz, float("nan")), torch.full_like(x, float("nan"))
    mr, dw, db = torch.empty(n, groups, 2, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.lamp_group_norm_act_fwd(p, x, z, mr, ws)
    B.lamp_group_norm_act_bwd(p, dz, x, mr, dx, dw, db, ws)
    given = torch.empty_like(z)                                             # the same with the channels' sums given
    stats = torch.empty(n, c, 2, dtype=torch.float64, device="cuda")
    for i in range(n):
        xs = x[i].view(v, c).double()
        stats[i] = torch.stack([xs.sum(0), xs.square().sum(0)], 1)
    mr2 = torch.empty_like(mr)
    B.lamp_group_norm_act_fwd(p, x, given, mr2, None, stats)
    wd, bd = w.double(), b.double()
    sums = torch.zeros(4, c, dtype=torch.float64, device="cuda")
    for i in range(n):
        xs, gs = x[i].view(v, c).double(), dz[i].view(v, c).double()
        flat = xs.view(v, groups, -1)
        mean = flat.mean((0, 2))
        rstd = 1 / torch.sqrt((flat - mean[None, :, None]).square().mean((0, 2)) + 1e-5)
        for got in (mr[i].double(), mr2[i].double()):
            assert ((got[:, 0] - mean).abs() <= U * (mean.abs() + 600 / rstd)).all() and ((got[:, 1] / rstd - 1).abs() <= 304 * U).all()
        # z and the gradients against the statistics that were kept: t is off by 4 u (|w| |xhat| + |t| + |b|)
        ref, t, xh, dt, rdx, s = sample_reference(xs, gs, mr[i, :, 0].double(), mr[i, :, 1].double(), wd, bd, groups, name)
        e = 4 * U * (wd.abs() * xh.abs() + t.abs() + bd.abs())
        own = 8 * U * ref.abs() + (0 if zt is torch.float32 else 4 * U * t * t * ref.abs() + 2.0 ** -22 * t.abs())
        tol = 1.13 * e + own
        tol = tol + torch.finfo(zt).eps / 2 * (ref.abs() + tol)
        assert ((z[i].view(v, c).double() - ref).abs() <= tol).all()
        ref2 = sample_reference(xs, gs, mr2[i, :, 0].double(), mr2[i, :, 1].double(), wd, bd, groups, name)[0]
        assert ((given[i].view(v, c).double() - ref2).abs() <= tol + torch.finfo(zt).eps / 2 * (ref2 - ref).abs()).all()
        sure = t.abs() > e if name == "leaky_relu" else torch.ones_like(t, dtype=torch.bool)
        edt = gs.abs() * (0.8 * e + 2.0 ** -22 * (1 + t.abs()) + 8 * U * t * t)
        unsure = torch.where(sure, 0.0, gs.abs())
        mean_of = lambda a: a.view(v, groups, -1).mean((0, 2)).repeat_interleave(c // groups)                 # noqa: E731
        wa = wd.abs()
        e1, e2 = mean_of(wa * (300 * U * dt.abs() + edt + unsure)), mean_of(wa * (304 * U * (dt * xh).abs() + (edt + unsure) * xh.abs()))
        c1, c2 = mean_of((wd * dt).abs()), mean_of((wd * dt * xh).abs())
        tol = s * (wa * edt + e1 + xh.abs() * e2 + 8 * U * ((wd * dt).abs() + c1 + xh.abs() * c2))
        tol = tol + torch.finfo(xt).eps / 2 * (rdx.abs() + tol)
        bad = ((dx[i].view(v, c).double() - rdx).abs() > tol) | dx[i].view(v, c).isnan()
        assert not (bad & sure).any()
        sums += torch.stack([dt.sum(0), (dt * xh).sum(0), (300 * U * dt.abs() + edt + unsure).sum(0), (304 * U * (dt * xh).abs() + (edt + unsure) * xh.abs()).sum(0)])
    assert ((db.double() - sums[0]).abs() <= sums[2] + U * sums[0].abs()).all() and ((dw.double() - sums[1]).abs() <= sums[3] + U * sums[1].abs()).all()


# more groups in a chunk than the pass that applies finishes itself; more channels of a group; both kinds of finishing kernel
@pytest.mark.parametrize("shape", [(1, (6, 6, 6), 2048, 2048), (2, (5, 5, 5), 8192, 2), (3, (2, 3, 2), 600, 300), (2, (4, 4, 4), 6144, 24)], ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_given_sums(shape, types):
    n, dhw, c, groups = shape
    xt, zt = TYPES[types]
    r, x, w, b = case(shape, 2)
    tx = dev(x, xt)
    xs = tx.view(n, -1, c).double()
    stats = torch.stack([xs.sum(1), xs.square().sum(1)], 2).contiguous()
    p = B.group_norm(groups, dev(w), dev(b), "gelu")
    z, mr = torch.empty(x.shape, dtype=zt, device="cuda"), torch.empty(n, groups, 2, device="cuda")
    B.lamp_group_norm_act_fwd(p, tx, z, mr, None, stats)
    check_forward(z, mr, host(tx), w, b, shape, "gelu", 0.0, 1e-5, zt)
