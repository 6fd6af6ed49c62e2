"""Block norm on the GPU (forward, 8-bit output, backward, parameter gradients) against the fp64 oracle.

Tolerances.  A row of c channels is summed by at most 16 terms per thread and a tree, so a mean or a mean square is off by
at most 32 units of 2^-24 of the mean magnitude; the normalised value v^ then by at most 64 units of 2^-24 (1 + A) with
A = (max |v| + |mean|) / deviation of its row, its weighted value by two more.  NORM below is 128 units.  Backward adds one
more pass of the same kind over each row.  Sums over rows: N terms per chain, N <= rows per thread + 16, each rounding one unit
of the sum of magnitudes; the last step is fp64.  A stored bf16 adds 2^-8 of the value."""
import numpy as np
import pytest
import torch

from oracle import pointwise as P
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
NORM = 128 * 2.0 ** -24
TY = {"b": torch.bfloat16, "f": torch.float32}


def dev(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(dt)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, tol, dt, what):
    if dt is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4], np.broadcast_to(tol, ref.shape)[bad][:4])


def spread(v, rms, eps):
    """1 + A of every row, [rows, 1]."""
    mean = 0.0 if rms else v.mean(1, keepdims=True)
    sd = np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)
    return 1 + (np.abs(v).max(1, keepdims=True) + np.abs(mean)) / sd


class Case:
    def __init__(self, seed, n, rows, c, types, gate, params=True, eps=1e-5):
        r = self.r = np.random.default_rng(seed)
        self.n, self.rows, self.c, self.eps = n, rows, c, eps
        self.ts, self.tb = TY[types[0]], TY[types[1]]
        self.shape = (n, 1, 1, rows, c)
        vec = lambda mu, sd: (mu + sd * r.standard_normal(c)).astype(np.float32) if params else None       # noqa: E731
        self.post_w, self.post_b, self.pre_w, self.pre_b, self.res = vec(1, .3), vec(0, .3), vec(1, .3), vec(0, .3), vec(.7, .2)
        self.gate_kind = gate
        self.gate = r.standard_normal((n, c)).astype(np.float32) if gate == "sample" else None
        self.logits = self.tensor(self.tb, 2.0) if gate == "element" else None

    def tensor(self, dt, scale=1.0, shift=0.0):
        return dev(self.r.standard_normal(self.shape) * scale + shift, dt)

    def params(self, rms):
        f = lambda a: None if a is None else dev(a, torch.float32)                                          # noqa: E731
        return B.block_norm(rms=rms, eps=self.eps, post_w=f(self.post_w), post_b=f(self.post_b), pre_w=f(self.pre_w), pre_b=f(self.pre_b),
                            gate=f(self.gate), gate_logits=self.logits, res_scale=f(self.res))

    def flat(self, t):
        return host(t).reshape(-1, self.c)

    def gate_values(self):
        if self.gate is not None:
            return np.repeat(self.gate.astype(np.float64), self.rows, axis=0)
        return P.sigmoid(self.flat(self.logits)) if self.logits is not None else 1.0

    def v(self, name):
        a = getattr(self, name)
        return (0.0 if name.endswith("_b") else 1.0) if a is None else a.astype(np.float64)


SIZES = [(1, 1, 8), (2, 3, 24), (1, 70, 32), (3, 33, 64), (1, 19, 120), (2, 40, 128), (1, 9, 200), (2, 17, 256), (1, 21, 264), (2, 5, 512),
         (1, 6, 520), (2, 7, 1032), (1, 3, 2048), (1, 5, 4096), (2, 2, 8192), (2, 700, 32), (1, 2500, 320)]


@pytest.mark.parametrize("n,rows,c", SIZES)
@pytest.mark.parametrize("types,rms,gate", [("bb", False, "sample"), ("fb", True, "element"), ("ff", False, "none"), ("bb", True, "none"),
                                            ("ff", True, "sample"), ("bb", False, "element")])
def test_forward(n, rows, c, types, rms, gate):
    k = Case(rows + c, n, rows, c, types, gate, params=rows % 2 == 1)
    y, x = k.tensor(k.tb, 1.5, 0.4), k.tensor(k.ts, 2.0, -0.3)
    out, h = torch.full_like(x, float("nan")), torch.full(k.shape, float("nan"), dtype=k.tb, device="cuda")
    p = k.params(rms)
    B.lamp_block_norm_fwd(p, y, x, out, h)
    yy, xx = k.flat(y), k.flat(x)
    g = k.gate_values()
    branch = k.v("res") * g * P.norm(yy, k.v("post_w"), k.v("post_b"), rms, k.eps)[0]
    scale = np.abs(k.v("res") * g) * (np.abs(k.v("post_w")) + np.abs(k.v("post_b")))
    t = xx + branch
    close(k.flat(out), t, NORM * spread(yy, rms, k.eps) * scale + 2.0 ** -23 * np.abs(t), k.ts, "out")
    st = k.flat(out)                                                    # h is the norm of t as stored
    href, hat, _ = P.norm(st, k.v("pre_w"), k.v("pre_b"), rms, k.eps)
    tol = NORM * spread(st, rms, k.eps) * (np.abs(k.v("pre_w")) + np.abs(k.v("pre_b")))
    close(k.flat(h), href, tol, k.tb, "h")
    # each half on its own gives the same bits, and in place
    o2, h2, x2 = torch.empty_like(out), torch.empty_like(h), x.clone()
    B.lamp_block_norm_fwd(p, y, x, o2, None)
    B.lamp_block_norm_fwd(p, y, x2, x2, None)
    f = lambda a: None if a is None else dev(a, torch.float32)          # noqa: E731
    B.lamp_block_norm_fwd(B.block_norm(rms=rms, eps=k.eps, pre_w=f(k.pre_w), pre_b=f(k.pre_b)), None, out, None, h2)
    assert torch.equal(o2, out) and torch.equal(x2, out) and torch.equal(h2, h)
    # h in 8 bits: scales as exact as h in fp32, codes within half a step of the scaled value
    q = torch.full((n * rows, -(-c // 16) * 16 + 16), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full((-(-c // 128), n * rows + 3), -7.0, device="cuda")
    o2.fill_(0)
    B.lamp_block_norm_fwd(p, y, x, o2, None, B.fp8_operand(q, s, n * rows, c))
    assert torch.equal(o2, out)
    gq, gs = q.cpu().numpy(), s.cpu().numpy().astype(np.float64)
    assert (gq[:, c:] == 0x55).all() and (gs[:, n * rows:] == -7).all()
    back = P.dequantize(gq[:, :c], gs[:, :n * rows], False)
    for b in range(-(-c // 128)):
        sl = slice(b * 128, min(c, b * 128 + 128))
        amax = np.abs(href[:, sl]).max(1)
        np.testing.assert_array_less(np.abs(gs[b, :n * rows] - amax / 448), (np.broadcast_to(tol, href.shape)[:, sl].max(1) + 2.0 ** -22 * amax) / 448 + 1e-38)
        step = np.maximum(2.0 ** -4 * np.abs(href[:, sl]), 2.0 ** -10 * gs[b, :n * rows, None])
        assert (np.abs(back[:, sl] - href[:, sl]) <= step * 1.001 + 2 * np.broadcast_to(tol, href.shape)[:, sl]).all()
    # the same call without the pre-norm's stored h is bit for bit what the quantiser makes of an fp32 h
    if types == "ff":
        q2, s2 = torch.zeros_like(q), torch.zeros_like(s)
        B.lamp_fp8_quantize(h, B.fp8_operand(q2, s2, n * rows, c))
        assert torch.equal(q2[:, :c], q[:, :c]) and torch.equal(s2[:, :n * rows], s[:, :n * rows])


def run_backward(k, rms, y, t, dout, dh, want=True):
    p = k.params(rms)
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")         # noqa: E731
    g = dict(dpost_w=nan(k.c), dpost_b=nan(k.c), dpre_w=nan(k.c), dpre_b=nan(k.c), dres_scale=nan(k.c),
             dgate=nan(k.n, k.c) if k.gate is not None else None) if want else {}
    dx, dy = torch.full(k.shape, float("nan"), dtype=k.ts, device="cuda"), torch.full(k.shape, float("nan"), dtype=k.tb, device="cuda")
    dl = torch.full_like(dy, float("nan")) if k.logits is not None else None
    nbytes = B.lamp_block_norm_bwd_workspace_bytes(t, p)
    ws = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device="cuda") if want else None
    B.lamp_block_norm_bwd(p, y, t, dout, dh, dx, dy, ws[:nbytes] if want else None, dgate_logits=dl, **g)
    if want:
        assert (ws[nbytes:] == 0xFF).all()
    return dx, dy, dl, g


@pytest.mark.parametrize("n,rows,c", SIZES)
@pytest.mark.parametrize("types,rms,gate", [("bb", False, "sample"), ("fb", True, "element"), ("ff", False, "none"), ("bb", True, "none"),
                                            ("ff", True, "sample"), ("fb", False, "element")])
def test_backward(n, rows, c, types, rms, gate):
    k = Case(rows + c + 1, n, rows, c, types, gate, params=rows % 2 == 1)
    y, t = k.tensor(k.tb, 1.5, 0.4), k.tensor(k.ts, 2.0, -0.3)
    dout, dh = k.tensor(k.ts), k.tensor(k.tb)
    dx, dy, dl, g = run_backward(k, rms, y, t, dout, dh)
    yy, tt, go, gh = (k.flat(v) for v in (y, t, dout, dh))
    gate_v = k.gate_values()
    ref = P.block_norm_backward(yy, tt, go, gh, k.v("post_w"), k.v("post_b"), k.v("pre_w"), k.v("res"), gate_v, rms, k.eps)
    # magnitudes that the roundings scale with
    sd = lambda v: np.sqrt(((v - (0 if rms else v.mean(1, keepdims=True))) ** 2).mean(1, keepdims=True) + k.eps)       # noqa: E731
    a = np.abs(gh * k.v("pre_w"))
    At, Ay = spread(tt, rms, k.eps), spread(yy, rms, k.eps)
    e_dx = NORM * (np.abs(go) + At ** 2 * (a + a.max(1, keepdims=True)) / sd(tt))
    close(k.flat(dx), ref["dx"], e_dx, k.ts, "dx")
    rg = np.abs(k.v("res") * gate_v)
    b = rg * np.abs(k.v("post_w")) * np.ones_like(yy)
    e_b = b * (e_dx + NORM * np.abs(ref["dx"]))
    mag_b = b * np.abs(ref["dx"])
    e_dy = 2 * Ay ** 2 * (e_b + e_b.max(1, keepdims=True) + NORM * (mag_b + mag_b.max(1, keepdims=True))) / sd(yy)
    close(k.flat(dy), ref["dy"], e_dy, k.tb, "dy")
    if dl is not None:
        d = gate_v * (1 - gate_v)
        u = np.abs(P.norm(yy, k.v("post_w"), k.v("post_b"), rms, k.eps)[0]) + Ay
        close(k.flat(dl), ref["gate"] * d, np.abs(k.v("res")) * u * (e_dx + 4 * NORM * (np.abs(ref["dx"]) + Ay)), k.tb, "dgate_logits")
    chain = (rows * n + 16) * 2.0 ** -24
    et = e_dx * (Ay + 1) + (NORM * (Ay + At)) * (np.abs(ref["dx"]) + np.abs(gh))
    for name, key in (("dpost_w", "post_w"), ("dpost_b", "post_b"), ("dpre_w", "pre_w"), ("dpre_b", "pre_b"), ("dres_scale", "res_scale")):
        f = {"post_w": rg, "post_b": rg, "res_scale": np.abs(gate_v) * (np.abs(k.v("post_w")) + np.abs(k.v("post_b")))}.get(key, 1.0)
        tol = (np.abs(ref[key]) * chain + et * f).sum(0) + 2.0 ** -23 * np.abs(ref[key].sum(0))
        close(host(g[name]), ref[key].sum(0), tol, torch.float32, name)
    if k.gate is not None:
        per = ref["gate"].reshape(n, rows, c)
        f = (np.abs(k.v("res")) * (np.abs(k.v("post_w")) + np.abs(k.v("post_b"))) * np.ones_like(yy)).reshape(n, rows, c)
        close(host(g["dgate"]), per.sum(1), (np.abs(per) * chain + et.reshape(n, rows, c) * f).sum(1) + 2.0 ** -23 * np.abs(per.sum(1)), torch.float32, "dgate")
    # the same bits again, without parameter gradients, and with dx in place of dout
    dx2, dy2, _, g2 = run_backward(k, rms, y, t, dout, dh)
    assert torch.equal(dx2, dx) and torch.equal(dy2, dy) and all(torch.equal(g2[i], g[i]) for i in g if g[i] is not None)
    dx3, dy3, _, _ = run_backward(k, rms, y, t, dout, dh, want=False)
    assert torch.equal(dx3, dx) and torch.equal(dy3, dy)
    p = k.params(rms)
    B.lamp_block_norm_bwd(p, y, t, dout, dh, dout, dy3, dgate_logits=torch.empty_like(dl) if dl is not None else None)
    assert torch.equal(dout, dx)


@pytest.mark.parametrize("c", [16, 256, 512, 1040])
def test_backward_of_each_half_alone(c):
    k = Case(4, 2, 9, c, "fb", "none")
    k.res = None
    y, t = k.tensor(k.tb, 1.5, 0.4), k.tensor(k.ts, 2.0, -0.3)
    dout, dh = k.tensor(k.ts), k.tensor(k.tb)
    # post-norm alone: dt = dout
    dx, dy, _, g = run_backward(k, False, y, t, dout, None)
    assert torch.equal(dx, dout) and (g["dpre_w"] == 0).all() and (g["dpre_b"] == 0).all()
    zero = torch.zeros_like(dh)
    _, dyz, _, gz = run_backward(k, False, y, t, dout, zero)
    assert torch.equal(dyz, dy) and torch.equal(gz["dpost_w"], g["dpost_w"])
    # pre-norm alone
    p = B.block_norm(pre_w=dev(k.pre_w, torch.float32), pre_b=dev(k.pre_b, torch.float32))
    d1, d2 = torch.empty_like(t), torch.empty_like(t)
    pw, pb = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    ws = torch.empty(B.lamp_block_norm_bwd_workspace_bytes(t, p), dtype=torch.uint8, device="cuda")
    B.lamp_block_norm_bwd(p, None, t, dout, dh, d1, None, ws, dpre_w=pw, dpre_b=pb)
    full, _, _, g = run_backward(k, False, y, t, dout, dh)
    assert torch.equal(d1, full) and torch.equal(pw, g["dpre_w"]) and torch.equal(pb, g["dpre_b"])
    B.lamp_block_norm_bwd(p, None, t, None, dh, d2, None)               # nothing past the block
    ref = P.block_norm_backward(None, k.flat(t), None, k.flat(dh), None, None, k.v("pre_w"), None, None, False, k.eps)["dx"]
    tt, a = k.flat(t), np.abs(k.flat(dh) * k.v("pre_w"))
    close(k.flat(d2), ref, NORM * spread(tt, False, k.eps) ** 2 * (a + a.max(1, keepdims=True)), torch.float32, "dx")


def test_rows_that_are_constant_huge_or_not_finite():
    c = 64
    k = Case(6, 1, 40, c, "bb", "none", params=False, eps=0.0)
    x, y = k.tensor(k.ts), k.tensor(k.tb)
    k.eps = 1e-5
    y[0, 0, 0, 3] = 0.0                                                 # deviation 0: N = 0
    y[0, 0, 0, 4] = 5.0
    y[0, 0, 0, 5] *= 1e18                                               # squares stay inside fp32
    y[0, 0, 0, 6, 7] = float("nan")
    y[0, 0, 0, 7, 9] = float("inf")
    out, h = torch.empty_like(x), torch.empty_like(x)
    B.lamp_block_norm_fwd(k.params(False), y, x, out, h)
    o = out[0, 0, 0].float()
    assert torch.equal(o[3], x[0, 0, 0, 3].float()) and torch.equal(o[4], x[0, 0, 0, 4].float())
    assert torch.isnan(o[6]).all() and torch.isnan(o[7]).any()
    keep = [i for i in range(40) if i not in (6, 7)]
    assert torch.isfinite(o[keep]).all() and torch.isfinite(h[0, 0, 0].float()[keep]).all()
    # eps = 0 with rows past the end of the last CTA's share: nothing of them reaches the sums
    k.eps = 0.0
    for c in (16, 64, 200):
        k = Case(7, 1, 3, c, "ff", "none", params=False, eps=0.0)
        y, t, dout, dh = (k.tensor(torch.float32) for _ in range(4))
        dx, dy, _, g = run_backward(k, False, y, t, dout, dh)
        assert all(torch.isfinite(v).all() for v in (dx, dy, g["dpost_w"], g["dpre_w"], g["dres_scale"]))


def test_channel_slices_and_untouched_neighbours():
    k = Case(8, 2, 11, 40, "bb", "sample")
    wide = lambda v: torch.full((*k.shape[:4], 64), v, dtype=torch.bfloat16, device="cuda")          # noqa: E731
    y, x, dout, dh = (k.tensor(torch.bfloat16) for _ in range(4))
    out, h = torch.empty_like(x), torch.empty_like(x)
    p = k.params(False)
    B.lamp_block_norm_fwd(p, y, x, out, h)
    bufs = [wide(9.0) for _ in range(4)]
    for b, v in zip(bufs[:2], (y, x)):
        b[..., 8:48] = v
    s = [B.tensor(b, 40, 8) for b in bufs]
    # descriptors carry no torch tensor to check, so the parameters' sizes are taken from them
    B.lamp_block_norm_fwd(p, s[0], s[1], s[2], s[3])
    assert torch.equal(bufs[2][..., 8:48], out) and torch.equal(bufs[3][..., 8:48], h)
    for b in bufs:
        assert (b[..., :8] == 9).all() and (b[..., 48:] == 9).all()


def test_graph_replay_streams_and_many_samples():
    k = Case(9, 37, 5, 96, "bb", "sample")                              # more samples than the finish kernel's warps
    y, t, dout, dh = (k.tensor(torch.bfloat16) for _ in range(4))
    dx, dy, _, g = run_backward(k, True, y, t, dout, dh)
    p = k.params(True)
    ws = torch.empty(B.lamp_block_norm_bwd_workspace_bytes(t, p), dtype=torch.uint8, device="cuda")
    bufs = {n: torch.empty_like(v) for n, v in g.items()}
    dx2, dy2 = torch.empty_like(dx), torch.empty_like(dy)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        B.lamp_block_norm_bwd(p, y, t, dout, dh, dx2, dy2, ws, **bufs)
    for _ in range(2):
        for v in (dx2, dy2, *bufs.values()):
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dx2, dx) and torch.equal(dy2, dy) and all(torch.equal(bufs[n], g[n]) for n in g)
