"""Top-k distillation loss on logits of any size: classes masked with large negative values, rows far from zero.

Softmax depends on differences alone, so the bound must not grow with |z|.  Tolerances, in units of u = 2^-24, with d = (z - max z) / T:
an exponent is one difference and two products with constants that carry two roundings, off by at most 5 u |d| however many steps a
running maximum takes (their |d| add up to it); an exponential adds 4 u, at most 8 of them are multiplied; a sum adds one unit
per level, at most 64.  The sum of exponentials is then off by (96 + 5 sum_i q_i |d_i|) u relative, and
sum_i q_i |d_i| <= log c.  Hence for a probability
    e(d, c) = (112 + 5 log c + 5 |d|) u    relative,
the same for its log, and for the teacher's with k in the place of c.  A teacher's probability from a given log-sum takes
t / T - lse as it stands: 4 u (|t| / T + |lse|) more.  The log-sum itself is max z / T + log sum, 4 u |max z| / T more.  A loss sums
p (log p - log q) in parts of magnitude |log p| + |d| + log sum, at most 64 levels.  The gradient alone starts from the stored
log-sum: z / T - lse is formed with 2 u |z| / T + 4 u |z / T - lse|.  A stored bf16 adds 2^-8 of the value."""
import numpy as np
import pytest
import torch

from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def near(got, ref, tol, what):
    got, ref, tol = np.broadcast_arrays(got, ref, tol)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], tol[bad][:4])


def check(z, idx, t, temp, tlse=None):
    """z [rows, c] on the GPU, idx and t [rows, k] numpy: loss, log-sum and gradient of all three calls against 64 bits."""
    rows, c = z.shape
    k = idx.shape[1]
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()              # noqa: E731
    teacher = B.teacher_topk(dev(idx), dev(t), temp, dev(tlse))
    zt = z.view(1, 1, 1, rows, c)
    w = torch.linspace(0.25, 1.0, rows, device="cuda")
    nan = lambda *s, dt=torch.float32: torch.full(s, float("nan"), dtype=dt, device="cuda")              # noqa: E731
    ws = torch.empty(B.lamp_distill_topk_workspace_bytes(zt), dtype=torch.uint8, device="cuda")
    loss, lse, total, fused, two = nan(rows), nan(rows), nan(1), nan(*zt.shape, dt=z.dtype), nan(*zt.shape, dt=z.dtype)
    B.lamp_distill_topk_fwd(zt, teacher, w, loss, lse, total, ws)
    loss2 = nan(rows)
    B.lamp_distill_topk_fwd_bwd(zt, teacher, w, loss2, total, fused, ws)
    B.lamp_distill_topk_bwd(zt, teacher, w, lse, two)
    assert B.lamp_get_async_status() == 0
    # 64 bits
    s, g = z.double().cpu().numpy() / temp, w.double().cpu().numpy()[:, None] * temp
    top = s.max(1, keepdims=True)
    d = s - top
    ls = np.log(np.exp(d).sum(1, keepdims=True))
    q = np.exp(d - ls)
    tt = t.astype(np.float64) / temp
    if tlse is None:
        dt = tt - tt.max(1, keepdims=True)
        logp = dt - np.log(np.exp(dt).sum(1, keepdims=True))
        ep = (112 + 5 * np.log(k) + 5 * np.abs(dt)) * U
    else:
        logp = tt - tlse.astype(np.float64)[:, None]
        ep = (112 + 4 * np.abs(tt) + 4 * np.abs(tlse.astype(np.float64))[:, None]) * U
    p = np.exp(logp)
    live = p > 0
    es = (112 + 5 * np.log(c)) * U
    dk = np.take_along_axis(d, idx, 1)
    with np.errstate(invalid="ignore"):
        term = np.where(live, p * (logp - (dk - ls)), 0.0)
        mag = np.where(live, p * (np.abs(logp) + np.abs(dk) + ls + 1), 0.0)
        etol = temp ** 2 * np.where(live, mag * (ep + 64 * U) + p * (ep + es + 5 * np.abs(dk) * U), 0.0).sum(1)
    ref_lse = (top + ls)[:, 0]
    near(lse.double().cpu().numpy(), ref_lse, es + 4 * U * (np.abs(top[:, 0]) + np.abs(ref_lse)), "log-sum")
    ref = temp ** 2 * term.sum(1)
    near(loss.double().cpu().numpy(), ref, etol, "loss")
    assert torch.equal(loss, loss2)
    S = p.sum(1, keepdims=True)
    listed, elisted = np.zeros_like(q), np.zeros_like(q)
    for r in range(rows):
        np.add.at(listed[r], idx[r], p[r])
        np.add.at(elisted[r], idx[r], p[r] * (ep[r] + 8 * U))
    eS = np.where(live, p * ep, 0.0).sum(1, keepdims=True) + 64 * U * S

    def gradient(got, q, eq, what):
        ref = g * (q * S - listed)
        tol = g * (q * (S * (eq + 8 * U) + eS) + elisted) + 8 * U * np.abs(ref) + 1e-37
        if z.dtype is torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
        near(got.view(rows, c).double().cpu().numpy(), ref, tol, what)
    gradient(fused, q, es + 5 * np.abs(d) * U, "gradient with the loss")
    arg = s - lse.double().cpu().numpy()[:, None]
    gradient(two, np.exp(arg), (16 + 2 * np.abs(s) + 4 * np.abs(arg)) * U, "gradient alone")


# classes, entries: one thread per row in registers and in shared memory, one warp with short and with long lists, one CTA, clusters
FORMS = [(9, 3), (30, 20), (90, 4), (90, 30), (600, 5), (1000, 100), (1000, 140), (3000, 10), (3000, 300), (50000, 70), (140000, 33)]


def patterns(c, k):
    """Which classes are masked; the listed ones are 7 apart from c - 1 downwards and stay."""
    r = np.random.default_rng(c)
    m = [np.arange(c) < c * 3 // 4, np.arange(c) >= c // 4, r.random(c) < 0.9, np.arange(c) % 2 == 0, np.arange(c) != c // 2]
    return np.array(m)


def listed(rows, c, k):
    return np.broadcast_to((c - 1 - np.arange(k) * (7 if 7 * k < c else 1)).astype(np.int32), (rows, k)).copy()


@pytest.mark.parametrize("temp", [1.0, 2.0, 5.0, 8.0])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,k", FORMS)
def test_classes_masked_with_large_negative_values(c, k, dt, temp):
    values = [-1e4, -1e9, -1e10, -1e30, torch.finfo(dt).min]
    masks = patterns(c, k)
    r = np.random.default_rng(1)
    rows = len(values) * len(masks)
    idx = listed(rows, c, k)
    z = torch.from_numpy((2 * r.standard_normal((rows, c))).astype(np.float32)).cuda().to(dt)
    for i, v in enumerate(values):
        for j, m in enumerate(masks):
            m = m.copy()
            m[idx[0]] = False
            z[i * len(masks) + j, torch.from_numpy(m).cuda()] = v
    check(z, idx, (2 * r.standard_normal((rows, k))).astype(np.float32), temp)


@pytest.mark.parametrize("temp", [1.0, 1.5, 5.0])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,k", FORMS)
def test_rows_far_from_zero(c, k, dt, temp):
    """A row moved by a common offset, and rows whose classes all have one and the same large value (fused call: uniform)."""
    r = np.random.default_rng(2)
    shifts = [1e3, -1e3, 1e5, -1e5, 3e7]
    base = np.round(16 * 2 * r.standard_normal((len(shifts), c))) / 16        # fp32 holds the moved rows exactly up to 1e5
    z = (base + np.array(shifts)[:, None]).astype(np.float32)
    check(torch.from_numpy(z).cuda().to(dt), listed(len(shifts), c, k), (2 * r.standard_normal((len(shifts), k))).astype(np.float32), temp)


@pytest.mark.parametrize("temp", [1.0, 2.0, 5.0, 8.0])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,k", FORMS)
def test_rows_of_one_large_value_are_uniform(c, k, dt, temp):
    """Loss and gradient in one call (the stored log-sum of such a row cannot hold log c beside the value)."""
    values = [-1e4, -1e9, -1e10, -1e30, 1e10, 1e30, torch.finfo(dt).min, torch.finfo(dt).max]
    rows = len(values)
    r = np.random.default_rng(3)
    idx, t = listed(rows, c, k), (2 * r.standard_normal((rows, k))).astype(np.float32)
    z = torch.empty(rows, c, dtype=dt, device="cuda")
    for i, v in enumerate(values):
        z[i] = v
    zt = z.view(1, 1, 1, rows, c)
    loss, dz, w = torch.full((rows,), float("nan"), device="cuda"), torch.full_like(zt, float("nan")), torch.ones(rows, device="cuda")
    B.lamp_distill_topk_fwd_bwd(zt, B.teacher_topk(torch.from_numpy(idx).cuda(), torch.from_numpy(t).cuda(), temp), w, loss, None, dz)
    tt = t.astype(np.float64) / temp
    logp = tt - np.log(np.exp(tt).sum(1, keepdims=True))
    p = np.exp(logp)
    e = (112 + 5 * np.log(c) + 5 * np.abs(logp)) * U
    ref = temp ** 2 * (p * (logp + np.log(c))).sum(1)
    near(loss.double().cpu().numpy(), ref, temp ** 2 * (p * ((np.abs(logp) + np.log(c) + 1) * (e + 64 * U) + 2 * e)).sum(1), "loss")
    g, tol = np.full((rows, c), temp / c), np.full((rows, c), temp / c * (240 + 10 * np.log(c)) * U)
    for i in range(rows):
        g[i, idx[i]] -= temp * p[i]
        tol[i, idx[i]] += temp * p[i] * (e[i] + 8 * U)
    if dt is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(g) + tol)
    near(dz.view(rows, c).double().cpu().numpy(), g, tol, "gradient")


@pytest.mark.parametrize("temp", [1.0, 1.5, 5.0])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("c,k", FORMS + [(9, 8), (40, 32), (600, 32), (600, 128), (700, 512), (5000, 1000)])
def test_teacher_far_from_zero(c, k, tail, temp):
    """The teacher's logits moved by a common offset, masked with large negative values, or all of one value (then p = 1 / k)."""
    r = np.random.default_rng(4)
    t = (np.round(16 * 2 * r.standard_normal((12, k))) / 16).astype(np.float32)
    low = np.finfo(np.float32).min
    for i, v in enumerate([1e3, -1e3, 1e5, -1e5, 3e7]):
        t[i] += np.float32(v)
    t[5, : k // 2] = -1e9
    t[6, k // 2 + 1:] = -1e30
    t[7, ::2] = low
    tlse = None
    if tail:                                                             # the log-sum of the first eight and a tail
        tt = t.astype(np.float64) / temp
        tlse = (tt.max(1) + np.log(np.exp(tt - tt.max(1, keepdims=True)).sum(1)) + 0.3).astype(np.float32)
        t, tlse = t[:8], tlse[:8]
    else:
        t[8], t[9], t[10], t[11] = -1e9, -1e30, low, -low
    z = torch.from_numpy((2 * r.standard_normal((len(t), c))).astype(np.float32)).cuda()
    check(z, listed(len(t), c, k), t, temp, tlse)


@pytest.mark.parametrize("temp", [2.0 ** -60, 2.0 ** -20, 2.0 ** 20, 2.0 ** 60])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,k", FORMS)
def test_smallest_and_largest_temperatures(c, k, dt, temp):
    r = np.random.default_rng(5)
    z = torch.from_numpy((2 * temp * r.standard_normal((3, c))).astype(np.float32)).cuda().to(dt)
    check(z, listed(3, c, k), (2 * temp * r.standard_normal((3, k))).astype(np.float32), temp)
