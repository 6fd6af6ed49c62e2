"""Group norm with an activation on the GPU against the fp64 oracle, forward and backward.

Tolerances, u = 2^-24, a = |w| rstd, t the argument of the activation.
  Sums of a thread run about a value of its own data over at most 256 values in fp32, so a mean is off by at most 300 u of the spread (2 sd counted for |x - k|) and by its own rounding u |mean|; a variance by 600 u relative, rstd by half of that and its
  rounding:  e_t = u (a (2 |mean| + 600 sd + 304 |x - mean|) + 4 (|t| + |b|)).
  The slope of every activation is below 1.13; its own value is off by 8 u |z| (fp32: expf, erfcf, one product) or, for bf16 outputs, by
  8 u |z| + 4 u t^2 |z| (e^x without the correction of x log2 e) + 2^-22 |t| (the rational form of the normal distribution).  Then half a step of the type
  (eps / 2 relative).
  Backward, from given mean and rstd: t as above without the statistics' part; the derivative changes by at most 0.8 e_t, its own value is off by
  16 u + 4 u t^2 (fp32 without the square) or 2^-22 (1 + |t|) for bf16; where the leaky ReLU's t is within e_t of 0 either slope is right.
  Sums over the voxels: 300 u of the sum of magnitudes and the sum of the terms' errors."""
import numpy as np
import pytest
import torch

from oracle import group as G
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ACTS = [("none", 0.0), ("leaky_relu", 0.0), ("leaky_relu", 0.1), ("silu", 0.0), ("gelu", 0.0)]
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32), "f32_bf16": (torch.float32, torch.bfloat16)}
# n, (d, h, w), c, groups
SHAPES = [(1, (1, 1, 1), 8, 8), (2, (1, 1, 1), 16, 2), (1, (1, 1, 2), 24, 8), (3, (2, 3, 5), 24, 3), (2, (4, 4, 4), 512, 32), (1, (7, 9, 11), 40, 40),
          (2, (8, 8, 8), 320, 32), (1, (20, 21, 22), 32, 4), (4, (5, 5, 5), 64, 1), (1, (6, 5, 4), 2056, 8), (2, (3, 3, 3), 4096, 4096), (1, (33, 32, 31), 136, 17),
          (1, (2, 2, 2), 2064, 3), (70, (1, 2, 3), 8, 2),
          # too many voxels for a cluster
          (1, (26, 26, 26), 24, 3), (2, (20, 30, 31), 48, 2), (1, (21, 21, 21), 320, 32)]


def dev(a, dt=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(dt)


def host(t):
    return t.double().cpu().numpy()


def sliced(a, dt, pad, off):
    """Tensor of the values a [n, v, c] as channels off .. off + c of a wider buffer: (descriptor, buffer, view of the values)."""
    n, d, h, w, c = a.shape
    buf = torch.full((n, d, h, w, c + pad), 3.0, dtype=dt, device="cuda")
    buf[..., off:off + c] = dev(a, dt)
    return B.tensor(buf, c, off), buf, buf[..., off:off + c]


def untouched(buf, off, c):
    return bool((buf[..., :off] == 3).all() and (buf[..., off + c:] == 3).all())


def case(shape, seed, loc=0.3, spread=1.5):
    n, dhw, c, groups = shape
    r = np.random.default_rng(seed)
    x = (loc + spread * r.standard_normal((n, *dhw, c)) * np.exp(0.5 * r.standard_normal(c)))
    return r, x, (1 + 0.3 * r.standard_normal(c)).astype(np.float32), (0.2 * r.standard_normal(c)).astype(np.float32)


def per_channel(s, c):
    return np.repeat(s, c // s.shape[1], axis=1)[:, None, :]


def t_error(x, mean, rstd, w, b, eps, given):
    c = x.shape[-1]
    m, s = per_channel(mean, c), per_channel(rstd, c)
    a, d = np.abs(w) * s, np.abs(x - m)
    t = (x - m) * s * w + b
    sd = np.sqrt(np.maximum(1 / s ** 2 - eps, 0))
    stat = 0.0 if given else a * (2 * np.abs(m) + 600 * sd + 304 * d)
    return t, U * (stat + 4 * a * d + 4 * (np.abs(t) + np.abs(b)))


def check_forward(z, mr, x, w, b, shape, name, slope, eps, zt):
    n, dhw, c, groups = shape
    x = x.reshape(n, -1, c)
    ref, mean, rstd = G.group_norm_act_fwd(x, groups, w, b, name, slope, eps)
    t, e = t_error(x, mean, rstd, w, b, eps, False)
    own = 8 * U * np.abs(ref) + (0 if zt is torch.float32 else 4 * U * t * t * np.abs(ref) + 2.0 ** -22 * np.abs(t))
    tol = 1.13 * e + own
    tol = tol + torch.finfo(zt).eps / 2 * (np.abs(ref) + tol)
    got = host(z).reshape(n, -1, c)
    bad = ~(np.abs(got - ref) <= tol + 1e-38)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3], tol[bad][:3])
    got = host(mr).reshape(n, groups, 2)
    sd = np.sqrt(np.maximum(1 / rstd ** 2 - eps, 0))
    assert (np.abs(got[..., 0] - mean) <= U * (np.abs(mean) + 600 * sd) + 1e-38).all()
    assert (np.abs(got[..., 1] - rstd) <= 304 * U * rstd).all()


def check_backward(dx, dw, db, dz, x, mr, w, b, shape, name, slope, eps, xt):
    n, dhw, c, groups = shape
    x, dz = x.reshape(n, -1, c), dz.reshape(n, -1, c)
    mean, rstd = mr[..., 0], mr[..., 1]
    rdx, rdw, rdb = G.group_norm_act_bwd(dz, x, mean, rstd, w, b, name, slope)
    t, e = t_error(x, mean, rstd, w, b, eps, True)
    slope_, s = G.act(t, name, slope)[1], per_channel(rstd, c)
    dt, xh = dz * slope_, (x - per_channel(mean, c)) * s
    if name in ("none", "leaky_relu"):
        e_dt = np.abs(dz) * (2 * U * np.abs(slope_) + (abs(1 - slope) * (np.abs(t) <= e) if name == "leaky_relu" else 0))
    else:
        e_dt = np.abs(dz) * (0.8 * e + (16 * U * (1 + np.abs(t)) + 4 * U * t * t if xt is torch.float32 else 2.0 ** -22 * (1 + np.abs(t)) + 8 * U * t * t))
    sums = lambda v, ev: (300 * U * np.abs(v) + ev)                                                             # noqa: E731
    e_b, e_w = sums(dt, e_dt).sum(axis=(0, 1)), sums(dt * xh, e_dt * np.abs(xh) + 4 * U * np.abs(dt * xh)).sum(axis=(0, 1))
    for got, ref, tol in ((dw, rdw, e_w), (db, rdb, e_b)):
        if got is not None:
            bad = ~(np.abs(host(got) - ref) <= tol + U * np.abs(ref) + 1e-38)
            assert not bad.any(), (bad.sum(), host(got)[bad][:3], ref[bad][:3], tol[bad][:3])
    mean_of = lambda v: per_channel(v.reshape(n, -1, groups, c // groups).mean(axis=(1, 3)), c)                # noqa: E731
    aw = np.abs(w)
    c1, c2 = mean_of(np.abs(w * dt)), mean_of(np.abs(w * dt * xh))
    e1, e2 = mean_of(aw * sums(dt, e_dt)), mean_of(aw * sums(dt * xh, e_dt * np.abs(xh) + 4 * U * np.abs(dt * xh)))
    tol = s * (aw * e_dt + e1 + np.abs(xh) * e2 + 8 * U * (np.abs(w * dt) + c1 + np.abs(xh) * c2))
    tol = tol + torch.finfo(xt).eps / 2 * (np.abs(rdx) + tol)
    got = host(dx).reshape(n, -1, c)
    bad = ~(np.abs(got - rdx) <= tol + 1e-38)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], got[bad][:3], rdx[bad][:3], tol[bad][:3])


def scratch(p, x):
    return torch.full((B.lamp_group_norm_workspace_bytes(p, x),), 0xFF, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_forward_matches_oracle(shape, types):
    n, dhw, c, groups = shape
    xt, zt = TYPES[types]
    for i, (name, slope) in enumerate(ACTS):
        r, x, w, b = case(shape, i)
        vx, xb, xv = sliced(x, xt, 8 * (i % 3), 8 * (i % 2) * (i % 3 > 0))
        vz, zb, zv = sliced(np.zeros_like(x), zt, 16, 8)
        mr = torch.full((n, groups, 2), float("nan"), device="cuda")
        eps = [1e-5, 0.1][i % 2]
        p = B.group_norm(groups, dev(w) if i != 1 else None, dev(b) if i != 2 else None, name, slope, eps)
        B.lamp_group_norm_act_fwd(p, vx, vz, mr, scratch(p, vx))
        check_forward(zv, mr, host(xv), w if i != 1 else np.ones(c), b if i != 2 else np.zeros(c), shape, name, slope, eps, zt)
        assert untouched(zb, 8, c)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_backward_matches_oracle(shape, types):
    n, dhw, c, groups = shape
    xt, zt = TYPES[types]
    for i, (name, slope) in enumerate(ACTS):
        r, x, w, b = case(shape, 10 + i)
        vx, _, xv = sliced(x, xt, 8 * (i % 3), 8 * (i % 2) * (i % 3 > 0))
        vg, _, gv = sliced(r.standard_normal(x.shape), zt, 8, 8)
        vd, db_, dv = sliced(np.zeros_like(x), xt, 24, 16)
        mean, rstd = G.statistics(host(xv).reshape(n, -1, c), groups, 1e-5)
        mr = dev(np.stack([mean, rstd], 2))
        p = B.group_norm(groups, dev(w) if i != 1 else None, dev(b) if i != 2 else None, name, slope, 1e-5)
        dw, db = (torch.full((c,), float("nan"), device="cuda") if i != k else None for k in (3, 4))
        B.lamp_group_norm_act_bwd(p, vg, vx, mr, vd, dw, db, scratch(p, vx))
        check_backward(dv, dw, db, host(gv), host(xv), host(mr), w if i != 1 else np.ones(c), b if i != 2 else np.zeros(c), shape, name, slope, 1e-5, xt)
        assert untouched(db_, 16, c)


def test_more_channels_than_a_cta_holds():
    shape = (1, (26, 25, 26), 2064, 2064)
    n, dhw, c, groups = shape
    r, x, w, b = case(shape, 9)
    tx, tg = dev(x, torch.bfloat16), dev(r.standard_normal(x.shape), torch.bfloat16)
    z, dx, mr = torch.empty_like(tx), torch.empty_like(tx), torch.empty(n, groups, 2, device="cuda")
    dw, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    p = B.group_norm(groups, dev(w), dev(b), "leaky_relu", 0.1)
    ws = scratch(p, tx)
    B.lamp_group_norm_act_fwd(p, tx, z, mr, ws)
    check_forward(z, mr, host(tx), w, b, shape, "leaky_relu", 0.1, 1e-5, torch.bfloat16)
    B.lamp_group_norm_act_bwd(p, tg, tx, mr, dx, dw, db, ws)
    check_backward(dx, dw, db, host(tg), host(tx), host(mr), w, b, shape, "leaky_relu", 0.1, 1e-5, torch.bfloat16)


@pytest.mark.parametrize("loc,spread", [(300.0, 0.01), (-1e4, 1.0), (0.0, 1e-3), (1e15, 1e13)])
def test_data_far_from_zero(loc, spread):
    shape = (2, (9, 10, 11), 48, 6)
    r, x, w, b = case(shape, 3, loc, spread)
    tx = dev(x)
    z, mr = torch.empty_like(tx), torch.empty(2, 6, 2, device="cuda")
    p = B.group_norm(6, dev(w), dev(b), "silu", 0.0, 0.0)
    B.lamp_group_norm_act_fwd(p, tx, z, mr, scratch(p, tx))
    check_forward(z, mr, host(tx), w, b, shape, "silu", 0.0, 0.0, torch.float32)


def test_one_outlier_at_the_start_of_every_group():
    shape = (1, (16, 16, 16), 32, 4)
    r, x, w, b = case(shape, 4)
    x[0, 0, 0, 0] = 1e4
    tx = dev(x)
    z, mr = torch.empty_like(tx), torch.empty(1, 4, 2, device="cuda")
    p = B.group_norm(4, dev(w), dev(b), "none")
    B.lamp_group_norm_act_fwd(p, tx, z, mr, scratch(p, tx))
    # a thread's shift is then up to 1e4 away from its other values: relative to the group's deviation (156) the spread is 64 times the 2 sd
    # that the general bound counts for it
    mean, rstd = G.statistics(host(tx).reshape(1, -1, 32), 4, 1e-5)
    assert (np.abs(host(mr)[..., 0] - mean) <= 64 * 300 * U / rstd + U * np.abs(mean)).all() and (np.abs(host(mr)[..., 1] / rstd - 1) <= 64 * 64 * 304 * U).all()


def test_constant_groups_and_zero_deviation():
    tx = torch.full((1, 2, 2, 2, 16), 7.25, device="cuda")
    z, mr = torch.empty_like(tx), torch.empty(1, 2, 2, device="cuda")
    b = torch.linspace(-1, 1, 16, device="cuda")
    p = B.group_norm(2, None, b, "none", 0.0, 1e-4)
    B.lamp_group_norm_act_fwd(p, tx, z, mr, scratch(p, tx))
    assert torch.equal(z, b.expand_as(z)) and (mr[..., 0] == 7.25).all() and torch.allclose(mr[..., 1], torch.tensor(100.0, device="cuda"), rtol=1e-6)


@pytest.mark.parametrize("name,slope", ACTS)
def test_values_that_are_not_finite_stay_in_their_group(name, slope):
    for bad in (float("nan"), float("inf")):
        tx = torch.randn(2, 3, 4, 5, 32, device="cuda")
        clean = tx.clone()
        tx[1, 2, 3, 4, 9] = bad
        p = B.group_norm(4, None, None, name, slope)
        out = []
        for t in (tx, clean):
            z, mr = torch.empty_like(t), torch.empty(2, 4, 2, device="cuda")
            B.lamp_group_norm_act_fwd(p, t, z, mr, scratch(p, t))
            out.append(z)
        z, ref = out
        assert z[1, ..., 8:16].isnan().all()
        z[1, ..., 8:16] = ref[1, ..., 8:16]
        assert torch.equal(z, ref)


def test_statistics_of_a_convolution():
    r = np.random.default_rng(8)
    n, d, c = 2, 12, 32
    x, wt = dev(r.standard_normal((n, d, d, d, 16)), torch.bfloat16), dev(r.standard_normal((27, c, 16)) * 0.05, torch.bfloat16)
    y, stats = torch.empty(n, d, d, d, c, device="cuda"), torch.zeros(n, c, 2, dtype=torch.float64, device="cuda")
    desc = B.conv_desc(16, c)
    ws = torch.empty(max(256, B.lamp_conv3d_workspace_bytes(desc, x, B.PASS_FWD)), dtype=torch.uint8, device="cuda")
    B.lamp_conv3d_fwd(desc, x, wt, None, y, stats, ws)
    w, b = (1 + 0.3 * r.standard_normal(c)).astype(np.float32), (0.2 * r.standard_normal(c)).astype(np.float32)
    p = B.group_norm(8, dev(w), dev(b), "gelu")
    for zt in (torch.float32, torch.bfloat16):
        z, mr = torch.empty(y.shape, dtype=zt, device="cuda"), torch.empty(n, 8, 2, device="cuda")
        B.lamp_group_norm_act_fwd(p, y, z, mr, None, stats)
        check_forward(z, mr, host(y), w, b, (n, (d, d, d), c, 8), "gelu", 0.0, 1e-5, zt)


@pytest.mark.parametrize("name", ["leaky_relu", "silu"])
@pytest.mark.parametrize("shape", [(2, (4, 5, 6), 64, 8), (1, (40, 40, 40), 64, 4)], ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_in_place_equals_out_of_place_and_repeats(name, shape, dt):
    n, dhw, c, groups = shape
    r, x, w, b = case(shape, 1)
    tx, tg = dev(x, dt), dev(r.standard_normal(x.shape), dt)
    p = B.group_norm(groups, dev(w), dev(b), name, 0.2)
    ws = scratch(p, tx)
    z, mr, mr2 = torch.empty_like(tx), torch.empty(n, groups, 2, device="cuda"), torch.empty(n, groups, 2, device="cuda")
    B.lamp_group_norm_act_fwd(p, tx, z, mr, ws)
    own = tx.clone()
    B.lamp_group_norm_act_fwd(p, own, own, mr2, ws)
    assert torch.equal(own, z) and torch.equal(mr, mr2)
    res = []
    for alias in (None, "dz", "x"):
        a, g = tx.clone(), tg.clone()
        dx = torch.empty_like(tx) if alias is None else g if alias == "dz" else a
        dw, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        B.lamp_group_norm_act_bwd(p, g, a, mr, dx, dw, db, ws)
        res.append((dx.clone(), dw, db))
    for other in res[1:]:
        assert all(torch.equal(u, v) for u, v in zip(res[0], other))


@pytest.mark.parametrize("shape", [(2, (4, 5, 6), 64, 8), (1, (48, 48, 48), 64, 4)], ids=str)
def test_on_a_side_stream_and_in_graphs_that_share_scratch(shape):
    n, dhw, c, groups = shape
    r, x, w, b = case(shape, 2)
    tx, tg = dev(x, torch.bfloat16), dev(r.standard_normal(x.shape), torch.bfloat16)
    p = B.group_norm(groups, dev(w), dev(b), "gelu")
    ws = scratch(p, tx)
    z, dx = torch.empty_like(tx), torch.empty_like(tx)
    mr, dw, db = torch.empty(n, groups, 2, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")

    def run():
        B.lamp_group_norm_act_fwd(p, tx, z, mr, ws)
        B.lamp_group_norm_act_bwd(p, tg, tx, mr, dx, dw, db, ws)
    run()
    ref = [t.clone() for t in (z, mr, dx, dw, db)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        run()
    st.synchronize()
    assert all(torch.equal(a, t) for a, t in zip(ref, (z, mr, dx, dw, db)))
    graphs = []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run()
    for g in graphs * 2:
        z.zero_(), dx.zero_(), dw.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(ref, (z, mr, dx, dw, db)))


def test_no_voxels():
    e = torch.empty(0, 2, 2, 2, 16, device="cuda")
    p = B.group_norm(4)
    dw, db = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    B.lamp_group_norm_act_fwd(p, e, e.clone(), torch.empty(0, 4, 2, device="cuda"))
    B.lamp_group_norm_act_bwd(p, e.clone(), e, torch.empty(0, 4, 2, device="cuda"), e.clone(), dw, db)
    assert (dw == 0).all() and (db == 0).all()


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(2, 1, 1, 4, 16, device="cuda")
    p, mr = B.group_norm(4, torch.ones(16, device="cuda")), torch.empty(2, 4, 2, device="cuda")
    ws = scratch(p, x)
    for call in (lambda: B.lamp_group_norm_act_fwd(B.group_norm(4, torch.ones(8, device="cuda")), x, x, mr, ws),
                 lambda: B.lamp_group_norm_act_fwd(p, x, x, mr[:1], ws),
                 lambda: B.lamp_group_norm_act_fwd(p, x, x, mr, ws, torch.zeros(2, 16, 2, device="cuda")),
                 lambda: B.lamp_group_norm_act_bwd(p, x, x, mr, x, torch.empty(8, device="cuda"), None, ws),
                 lambda: B.lamp_group_norm_act_fwd(p, x.half(), x, mr, ws)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.LampError):
        B.lamp_group_norm_act_fwd(p, x, x, mr, ws[:16])
