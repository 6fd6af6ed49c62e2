"""The operators together, as a program uses them: a block of group norm + SiLU and a channel-mixing layer in 4 bits, trained with
gradients clipped by their global norm - eager, on a side stream and as a replayed graph.

Forward z = silu(gn(x)), y = z W^T + bias; backward from dy: dz = dy W, dW = dy^T z, and the group norm's gradients; then the norm of all gradients and
the update with the clipping factor.  Each step is held against fp64 with the inputs that the GPU stored for it, so that every
tolerance is that of one operator (their derivations are in the operators' own tests)."""
import math

import numpy as np
import pytest
import torch

from oracle import fp4 as Q
from oracle import group as G
from oracle import optim
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
N, DHW, CIN, COUT, GROUPS = 2, (5, 6, 7), 72, 40, 9
V = N * DHW[0] * DHW[1] * DHW[2]
MAX_NORM, LR, ALPHA, EPS = 0.5, 1e-2, 0.9, 1e-6


def host(t):
    return t.double().cpu().numpy()


def operand(rows, k, block):
    g = torch.full((1,), 2.0 ** -6, device="cuda") if block == 16 else None
    q = torch.zeros(rows, -(-(-(-k // 2)) // 16) * 16, dtype=torch.uint8, device="cuda")
    return B.fp4_operand(q, torch.zeros(Q.scale_bytes(rows, k, block), dtype=torch.uint8, device="cuda"), rows, k, block, g)


class Block:
    def __init__(self, block, seed):
        r = np.random.default_rng(seed)
        t = lambda *s, dt=torch.float32, scale=1.0, loc=0.0: torch.from_numpy(loc + scale * r.standard_normal(s)).to(dt).cuda()          # noqa: E731
        e = lambda *s, dt=torch.float32: torch.full(s, float("nan"), dtype=dt, device="cuda")                                              # noqa: E731
        bf = torch.bfloat16
        self.block = block
        self.x, self.dy = t(N, *DHW, CIN, dt=bf, scale=2.0, loc=0.5), t(N, *DHW, COUT, dt=bf, scale=0.1)
        self.w32, self.bias = t(1, 1, 1, COUT, CIN, scale=0.1), t(COUT)
        self.w16, self.gw, self.gb = self.w32.to(bf), t(CIN, scale=0.2, loc=1.0), t(CIN, scale=0.1)
        self.v = [torch.zeros_like(p) for p in (self.w32, self.gw, self.gb)]
        self.z, self.dz, self.dx = e(N, *DHW, CIN, dt=bf), e(N, *DHW, CIN, dt=bf), e(N, *DHW, CIN, dt=bf)
        self.y, self.mr = e(N, *DHW, COUT, dt=bf), e(N, GROUPS, 2)
        self.dw, self.dgw, self.dgb = e(1, 1, 1, COUT, CIN), e(CIN), e(CIN)
        self.ops = {k: operand(*s, block) for k, s in dict(z=(V, CIN), w=(COUT, CIN), dy=(V, COUT), wt=(CIN, COUT), dyt=(COUT, V), zt=(CIN, V)).items()}
        self.p = B.group_norm(GROUPS, self.gw, self.gb, "silu")
        self.grads = B.grad_list([self.dw, self.dgw, self.dgb])
        self.norm, self.factor = e(1), e(1)
        self.ws = torch.empty(max(B.lamp_group_norm_workspace_bytes(self.p, self.x), B.lamp_grad_norm_workspace_bytes(self.grads)), dtype=torch.uint8, device="cuda")

    def step(self):
        o = self.ops
        B.lamp_group_norm_act_fwd(self.p, self.x, self.z, self.mr, self.ws)
        B.lamp_fp4_quantize(self.z, o["z"])
        B.lamp_fp4_quantize(self.w16, o["w"])
        B.lamp_gemm_fp4(o["z"], o["w"], self.y, self.bias)
        B.lamp_fp4_quantize(self.dy, o["dy"])
        B.lamp_fp4_quantize(self.w16, o["wt"], True)
        B.lamp_gemm_fp4(o["dy"], o["wt"], self.dz)
        B.lamp_fp4_quantize(self.dy, o["dyt"], True)
        B.lamp_fp4_quantize(self.z, o["zt"], True)
        B.lamp_gemm_fp4(o["dyt"], o["zt"], self.dw)
        B.lamp_group_norm_act_bwd(self.p, self.dz, self.x, self.mr, self.dx, self.dgw, self.dgb, self.ws)
        B.lamp_grad_norm(self.grads, MAX_NORM, self.norm, self.factor, self.ws)
        for g, p, v, p16 in ((self.dw, self.w32, self.v[0], self.w16), (self.dgw, self.gw, self.v[1], None), (self.dgb, self.gb, self.v[2], None)):
            B.lamp_rmsprop_step_scaled(g, self.factor, p, v, p16, LR, ALPHA, EPS)

    def state(self):
        return {k: getattr(self, k).clone() for k in ("z", "mr", "y", "dz", "dw", "dx", "dgw", "dgb", "norm", "factor", "w32", "w16", "gw", "gb")}


def dequantized(x, transpose, block):
    x = x.astype(np.float32)
    return Q.dequantize(*Q.quantize(x.T if transpose else x, block, 2.0 ** -6 if block == 16 else 1.0), block, 2.0 ** -6 if block == 16 else 1.0)


def product_close(got, a, b, bias, bf16):
    ref = a @ b.T + (0 if bias is None else bias)
    tol = (76 + a.shape[1] // 64) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -23 * (0 if bias is None else np.abs(bias))
    tol = tol + (2.0 ** -8 * (np.abs(ref) + tol) if bf16 else 0)
    assert (np.abs(got - ref) <= tol).all()


def check_step(b, before):
    """One step's results against fp64, from the parameters it started with (`before`) and what it stored."""
    x, z, dy, dz = (host(t).reshape(N, -1, t.shape[-1]) for t in (b.x, b.z, b.dy, b.dz))
    gw, gb, w16 = before["gw"], before["gb"], before["w16"].reshape(COUT, CIN)
    ref, mean, rstd = G.group_norm_act_fwd(x, GROUPS, gw, gb, "silu")
    t = G.normalise(x, mean, rstd) * gw + gb
    assert (np.abs(z - ref) <= 2.0 ** -8 * np.abs(ref) + 2000 * U * (1 + np.abs(t))).all()
    zf, dyf, dzf = (a.reshape(V, -1) for a in (z, dy, dz))
    k = b.block
    product_close(host(b.y).reshape(V, COUT), dequantized(zf, False, k), dequantized(w16, False, k), host(b.bias), True)
    product_close(dzf, dequantized(dyf, False, k), dequantized(w16, True, k), None, True)
    product_close(host(b.dw).reshape(COUT, CIN), dequantized(dyf, True, k), dequantized(zf, True, k), None, False)
    mr = host(b.mr)
    rdx, rdw, rdb = G.group_norm_act_bwd(dz, x, mr[..., 0], mr[..., 1], gw, gb, "silu")
    xh = G.normalise(x, mr[..., 0], mr[..., 1])
    s = np.repeat(mr[..., 1], CIN // GROUPS, axis=1)[:, None, :]
    big = np.abs(gw * dz).max()
    assert (np.abs(host(b.dx).reshape(x.shape) - rdx) <= 2.0 ** -8 * np.abs(rdx) + 4000 * U * s * big * (1 + np.abs(xh))).all()
    for got, want, mag in ((b.dgw, rdw, np.abs(dz * xh).sum(axis=(0, 1))), (b.dgb, rdb, np.abs(dz).sum(axis=(0, 1)))):
        assert (np.abs(host(got) - want) <= 4000 * U * mag).all()
    norm, factor, _ = G.clip([host(g) for g in (b.dw, b.dgw, b.dgb)], MAX_NORM)
    assert abs(b.norm.item() - norm) <= 5 * U * norm and abs(b.factor.item() - factor) <= 6 * U * factor and factor < 1
    for name, g, v in (("w32", b.dw, 0), ("gw", b.dgw, 1), ("gb", b.dgb, 2)):
        w, nv, _ = optim.rmsprop_step(before[name], host(g) * b.factor.item(), before["v"][v], LR, ALPHA, EPS)
        # fp32: the weight's rounding, and a step of at most lr / sqrt(1 - alpha) off by a few roundings
        assert (np.abs(host(getattr(b, name)) - w) <= U * np.abs(w) + 16 * U * LR / math.sqrt(1 - ALPHA)).all()
    assert torch.equal(b.w16, b.w32.to(torch.bfloat16))


def parameters(b):
    return dict(gw=host(b.gw), gb=host(b.gb), w32=host(b.w32), w16=host(b.w16), v=[host(v) for v in b.v])


@pytest.mark.parametrize("block", [32, 16])
def test_steps_of_a_block_match_fp64_step_by_step(block):
    b = Block(block, 1)
    for _ in range(3):
        before = parameters(b)
        b.step()
        assert B.lamp_get_async_status() == 0
        check_step(b, before)


@pytest.mark.parametrize("block", [32, 16])
def test_side_stream_and_replayed_graph_give_the_same_bits(block):
    eager, side, graph = (Block(block, 2) for _ in range(3))
    want = []
    for _ in range(3):
        eager.step()
        want.append(eager.state())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        for i in range(3):
            side.step()
            got = side.state()
            st.synchronize()
            assert all(torch.equal(got[k], want[i][k]) for k in got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graph.step()
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        got = graph.state()
        assert all(torch.equal(got[k], want[i][k]) for k in got)


def test_two_streams_at_once():
    """Two blocks on two streams share nothing and disturb nothing."""
    alone = [Block(32, 3), Block(16, 4)]
    for b in alone:
        for _ in range(5):
            b.step()
    torch.cuda.synchronize()
    both, streams = [Block(32, 3), Block(16, 4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for b, s in zip(both, streams):
            with torch.cuda.stream(s):
                b.step()
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        sa, sb = a.state(), b.state()
        assert all(torch.equal(sa[k], sb[k]) for k in sa)
