"""The same operators where element offsets pass 2^31: sampled against fp64, at both ends of the tensors."""
import math

import numpy as np
import pytest
import torch

from oracle import fp4 as Q
from oracle import group as G
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


def ends(n, k=2000):
    r = np.random.default_rng(0)
    return np.unique(np.concatenate([np.arange(64), n - 1 - np.arange(64), r.integers(0, n, k)]))


@pytest.mark.parametrize("name", ["silu", "leaky_relu"])
def test_group_norm(name):
    v, c, groups = (1 << 27) + 12345, 16, 2
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1, 1, 1, v, c, dtype=torch.bfloat16, device="cuda")
    for i in range(0, v, 1 << 24):
        x[0, 0, 0, i:i + (1 << 24)].normal_(0.5, 2.0, generator=g)
    assert x.numel() > 1 << 31
    w, b = torch.linspace(0.5, 1.5, c, device="cuda"), torch.linspace(-0.3, 0.3, c, device="cuda")
    p = B.group_norm(groups, w, b, name, 0.1)
    z, mr = torch.empty_like(x), torch.empty(1, groups, 2, device="cuda")
    ws = torch.empty(B.lamp_group_norm_workspace_bytes(p, x), dtype=torch.uint8, device="cuda")
    B.lamp_group_norm_act_fwd(p, x, z, mr, ws)
    s = torch.zeros(groups, 2, dtype=torch.float64, device="cuda")
    for i in range(0, v, 1 << 24):
        d = x[0, 0, 0, i:i + (1 << 24)].double().view(-1, groups, c // groups)
        s += torch.stack([d.sum((0, 2)), (d * d).sum((0, 2))], 1)
    m = v * (c // groups)
    mean = (s[:, 0] / m).cpu().numpy()
    rstd = 1 / np.sqrt((s[:, 1] / m).cpu().numpy() - mean ** 2 + 1e-5)
    got = mr[0].double().cpu().numpy()
    # a thread's sums of at most 256 values, as in the operator's own tests
    assert (np.abs(got[:, 0] - mean) <= U * (np.abs(mean) + 600 * 2.0)).all() and (np.abs(got[:, 1] / rstd - 1) <= 304 * U).all()
    at = torch.from_numpy(ends(v)).cuda()
    xs = x[0, 0, 0, at].double().cpu().numpy()[None]
    t = G.normalise(xs, got[None, :, 0], got[None, :, 1]) * w.double().cpu().numpy() + b.double().cpu().numpy()
    ref = G.act(t, name, 0.1)[0]
    assert (np.abs(z[0, 0, 0, at].double().cpu().numpy()[None] - ref) <= 2.0 ** -8 * np.abs(ref) + 64 * U * (1 + np.abs(t))).all()
    dz = z
    dz.copy_(x.flip(4))
    dw, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    dx = torch.empty_like(x)
    B.lamp_group_norm_act_bwd(p, dz, x, mr, dx, dw, db, ws)
    # sums over everything in fp64, a slice at a time
    tot = torch.zeros(4, c, dtype=torch.float64, device="cuda")
    mg, rg = (mr[0, :, i].double().repeat_interleave(c // groups) for i in (0, 1))
    for i in range(0, v, 1 << 24):
        xh = (x[0, 0, 0, i:i + (1 << 24)].double() - mg) * rg
        tt = xh * w + b
        sl = torch.sigmoid(tt) * (1 + tt * torch.sigmoid(-tt)) if name == "silu" else torch.where(tt > 0, 1.0, 0.1)
        dt = dz[0, 0, 0, i:i + (1 << 24)].double() * sl
        tot += torch.stack([dt.sum(0), (dt * xh).sum(0), dt.abs().sum(0), (dt * xh).abs().sum(0)])
    tot = tot.cpu().numpy()
    assert (np.abs(db.double().cpu().numpy() - tot[0]) <= 400 * U * tot[2]).all() and (np.abs(dw.double().cpu().numpy() - tot[1]) <= 400 * U * tot[3]).all()
    wn = w.double().cpu().numpy()
    level, along = ((wn * tot[i]).reshape(groups, -1).sum(1) / m for i in (0, 1))
    xh = G.normalise(xs, got[None, :, 0], got[None, :, 1])
    dzs = dz[0, 0, 0, at].double().cpu().numpy()[None]
    sl = G.act(t, name, 0.1)[1]
    sure = (np.abs(t) > 1e-5) if name == "leaky_relu" else np.ones_like(t, bool)
    per = lambda a: np.repeat(a, c // groups)                                                                     # noqa: E731
    ref = (dzs * sl * wn - per(level) - xh * per(along)) * per(got[:, 1])
    bad = np.abs(dx[0, 0, 0, at].double().cpu().numpy()[None] - ref) > 2.0 ** -8 * np.abs(ref) + 400 * U * (1 + np.abs(dzs)) * (1 + np.abs(xh))
    assert not (bad & sure).any()


def test_clipping():
    n = (1 << 31) + 4097
    g = torch.empty(n, dtype=torch.bfloat16, device="cuda").fill_(0.5)
    g[-1], g[0] = 3.0, -2.0
    lst = B.grad_list([g[1:]])                                             # off every boundary
    norm, factor = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(B.lamp_grad_norm_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
    want = math.sqrt((n - 2) * 0.25 + 9.0)
    B.lamp_grad_clip(lst, want / 2, norm, factor, ws)
    assert abs(norm.item() - want) <= 5 * U * want and abs(factor.item() - 0.5) <= 6 * U
    f = factor.item()
    assert g[0] == -2 and abs(g[-1].item() - 3 * f) <= 2.0 ** -8 * 3 * f
    for i in range(1, n - 1, 1 << 28):
        part = g[i:min(i + (1 << 28), n - 1)]
        assert (part == torch.tensor(0.5 * f).to(torch.bfloat16).item()).all()


@pytest.mark.parametrize("transpose", [False, True])
def test_quantiser_and_back(transpose):
    rows, c, block = (1 << 25) + 77, 72, 16
    x = torch.empty(1, 1, 1, rows, c, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    for i in range(0, rows, 1 << 22):
        x[0, 0, 0, i:i + (1 << 22)].normal_(0.0, 3.0, generator=g)
    assert x.numel() > 1 << 31
    r, k = (c, rows) if transpose else (rows, c)
    q = torch.zeros(r, -(-(-(-k // 2)) // 16) * 16, dtype=torch.uint8, device="cuda")
    s = torch.zeros(B.lamp_fp4_scale_bytes(r, k, block), dtype=torch.uint8, device="cuda")
    op = B.fp4_operand(q, s, r, k, block)
    B.lamp_fp4_quantize(x, op, transpose)
    y = torch.zeros_like(x)
    B.lamp_fp4_dequantize(op, y, transpose)
    if transpose:                                                           # blocks of 16 voxels
        for v0 in (0, 16 * ((rows // 16) // 2), 16 * (rows // 16)):
            xs = x[0, 0, 0, v0:v0 + 16].float().cpu().numpy().T
            np.testing.assert_array_equal(y[0, 0, 0, v0:v0 + 16].float().cpu().numpy().T, Q.dequantize(*Q.quantize(xs, block), block).astype(np.float32))
    else:
        at = torch.from_numpy(ends(rows, 300)).cuda()
        xs = x[0, 0, 0, at].float().cpu().numpy()
        np.testing.assert_array_equal(y[0, 0, 0, at].float().cpu().numpy(), Q.dequantize(*Q.quantize(xs, block), block).astype(np.float32))


@pytest.mark.parametrize("n", [2056, 2059])
def test_product(n):
    m, k, block = (1 << 20) + 131, 96, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    xa, xb = torch.randn(1, 1, 1, m, k, device="cuda", generator=g), torch.randn(1, 1, 1, n, k, device="cuda", generator=g)
    ops = []
    for x, rows in ((xa, m), (xb, n)):
        op = B.fp4_operand(torch.zeros(rows, 48, dtype=torch.uint8, device="cuda"), torch.zeros(B.lamp_fp4_scale_bytes(rows, k, block), dtype=torch.uint8, device="cuda"), rows, k, block)
        B.lamp_fp4_quantize(x, op)
        ops.append(op)
    y = torch.full((1, 1, 1, m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert y.numel() > 1 << 31
    B.lamp_gemm_fp4(ops[0], ops[1], y)
    assert B.lamp_get_async_status() == 0
    at = ends(m, 200)
    a = Q.dequantize(*Q.quantize(xa[0, 0, 0, torch.from_numpy(at).cuda()].cpu().numpy(), block), block)
    b = Q.dequantize(*Q.quantize(xb[0, 0, 0].cpu().numpy(), block), block)
    ref = a @ b.T
    tol = (76 + 1) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)
    got = y[0, 0, 0, torch.from_numpy(at).cuda()].double().cpu().numpy()
    assert (np.abs(got - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol)).all()
    for i in range(0, m, 1 << 17):
        assert not y[0, 0, 0, i:i + (1 << 17)].isnan().any()
