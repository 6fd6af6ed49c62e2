"""The per-voxel operators as they are used together: a channel-mixing residual block over a small volume, a class head and a
distillation loss, forward and backward, on the library's calls alone.

    h0 = N(x) in 8 bits,  y1 = h0 W1^T + b1,  y2 = q(y1) W2^T,  t = x + r g N(y2),  h = N(t) in 8 bits,  z = h Wz^T
    loss(z, teacher) and its gradient;  dh = q(dz) Wz,  (dt, dy2) = block norm backward,  dW2 = q(dy2)^T q(y1)^T,  dy1 = q(dy2) W2

End to end against the same chain in 64 bits with the oracle's own quantisation.  The two differ by bf16 roundings (at most
2^-8 of a value, about 2^-9 in the mean) after each of the at most 8 steps to an output, and where such a difference moves an
8-bit code to its neighbour: a share of about 2^-9 / 2^-4 of the codes moves by at most 2^-3 of its value, sqrt(1/32) 2^-3 = 2.2 %
of the norm per quantisation at the very most, 4 of them on the longest way, added in squares with the roundings: below 5 %."""
import numpy as np
import pytest
import torch

from oracle import pointwise as P
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
N, DHW, C, F, K, KT, EPS, T = 2, (3, 5, 7), 264, 520, 37, 6, 1e-5, 1.5
V = DHW[0] * DHW[1] * DHW[2]
R = N * V


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).float().numpy()


class Buffers:
    """Everything a program keeps: weights in both operand forms, activations, codes, gradients, scratch."""

    def __init__(self, seed):
        r = np.random.default_rng(seed)
        self.np = dict(x=bf(r.standard_normal((R, C))), w1=bf(r.standard_normal((F, C)) / C ** 0.5), w2=bf(r.standard_normal((C, F)) / F ** 0.5),
                       wz=bf(r.standard_normal((K, C)) / C ** 0.5 * 3), b1=0.3 * r.standard_normal(F).astype(np.float32),
                       nw=(1 + 0.2 * r.standard_normal((3, C))).astype(np.float32), nb=(0.1 * r.standard_normal((3, C))).astype(np.float32),
                       res=(0.5 + 0.1 * r.standard_normal(C)).astype(np.float32), gate=r.random((N, C)).astype(np.float32),
                       idx=r.integers(0, K, (R, KT)).astype(np.int32), tl=(2 * r.standard_normal((R, KT))).astype(np.float32),
                       weight=(r.random(R) / R).astype(np.float32))
        self.np["weight"][::9] = 0.0
        d = self.d = {k: torch.from_numpy(v).cuda() for k, v in self.np.items()}
        self.x = self.vol(C)
        self.x.view(R, C).copy_(d["x"])
        self.op = {}
        for name, w in (("w1", d["w1"]), ("w2", d["w2"]), ("wz", d["wz"])):
            src = w.to(torch.bfloat16).view(1, 1, 1, *w.shape)
            for tr in (False, True):
                o = self.operand(*(w.shape[::-1] if tr else w.shape), tile=True)
                B.lamp_fp8_quantize(src, o, tr)
                self.op[name, tr] = o
        self.h0, self.h, self.q1 = self.operand(R, C), self.operand(R, C), self.operand(R, F)
        self.qz, self.q2, self.q2t, self.q1t = self.operand(R, K8), self.operand(R, C), self.operand(C, R), self.operand(F, R)
        self.y1, self.y2, self.t, self.dt, self.dy2, self.dh, self.dy1 = self.vol(F), self.vol(C), self.vol(C), self.vol(C), self.vol(C), self.vol(C), self.vol(F)
        self.z, self.dz = self.vol(K8), torch.zeros((N, *DHW, K8), dtype=torch.bfloat16, device="cuda")
        self.dw2 = torch.empty((1, 1, 1, C, F), device="cuda")
        self.rows, self.loss = torch.empty(R, device="cuda"), torch.empty(1, device="cuda")
        self.grads = {n: torch.empty(C, device="cuda") for n in ("dpost_w", "dpost_b", "dpre_w", "dpre_b", "dres_scale")}
        self.grads["dgate"] = torch.empty(N, C, device="cuda")
        nw, nb = d["nw"], d["nb"]
        self.first = B.block_norm(pre_w=nw[0], pre_b=nb[0], eps=EPS)
        self.block = B.block_norm(eps=EPS, post_w=nw[1], post_b=nb[1], pre_w=nw[2], pre_b=nb[2], gate=d["gate"], res_scale=d["res"])
        self.ws = torch.empty(max(B.lamp_block_norm_bwd_workspace_bytes(self.t, self.block), B.lamp_distill_topk_workspace_bytes(self.z)),
                              dtype=torch.uint8, device="cuda")
        self.teacher = B.teacher_topk(d["idx"], d["tl"], T)

    def vol(self, c):
        return torch.empty((N, *DHW, c), dtype=torch.bfloat16, device="cuda")

    def operand(self, rows, k, tile=False):
        return B.fp8_operand(torch.zeros(rows, -(-k // 16) * 16, dtype=torch.uint8, device="cuda"),
                             torch.zeros(-(-k // 128), -(-rows // 128) if tile else rows, device="cuda"), rows, k, tile)

    def step(self):
        B.lamp_block_norm_fwd(self.first, None, self.x, None, None, self.h0)
        B.lamp_gemm_fp8(self.h0, self.op["w1", False], self.y1, self.d["b1"])
        B.lamp_fp8_quantize(self.y1, self.q1)
        B.lamp_gemm_fp8(self.q1, self.op["w2", False], self.y2)
        B.lamp_block_norm_fwd(self.block, self.y2, self.x, self.t, None, self.h)
        logits = B.tensor(self.z, K)                                     # 37 classes in a buffer 40 wide
        B.lamp_gemm_fp8(self.h, self.op["wz", False], logits)
        B.lamp_distill_topk_fwd_bwd(logits, self.teacher, self.d["weight"], self.rows, self.loss, B.tensor(self.dz, K), self.ws)
        B.lamp_fp8_quantize(self.dz, self.qz)                            # the three classes that are none carry zeros
        wzt = B.Fp8Operand(*(getattr(self.op["wz", True], f) for f, _ in B.Fp8Operand._fields_))
        qz = B.Fp8Operand(*(getattr(self.qz, f) for f, _ in B.Fp8Operand._fields_))
        qz.k = wzt.k = K
        B.lamp_gemm_fp8(qz, wzt, self.dh)
        B.lamp_block_norm_bwd(self.block, self.y2, self.t, None, self.dh, self.dt, self.dy2, self.ws, **self.grads)
        B.lamp_fp8_quantize(self.dy2, self.q2)
        B.lamp_gemm_fp8(self.q2, self.op["w2", True], self.dy1)
        B.lamp_fp8_quantize(self.dy2, self.q2t, True)
        B.lamp_fp8_quantize(self.y1, self.q1t, True)
        B.lamp_gemm_fp8(self.q2t, self.q1t, self.dw2)

    def outputs(self):
        return dict(t=self.t, z=self.z[..., :K], rows=self.rows, loss=self.loss, dt=self.dt, dy2=self.dy2, dy1=self.dy1, dw2=self.dw2, **self.grads)


K8 = 40


def reference(n):
    q = lambda a, tile=False: P.dequantize(*P.quantize(np.asarray(a, np.float32), tile), tile)            # noqa: E731
    f = {k: v.astype(np.float64) for k, v in n.items() if v.dtype == np.float32}
    nw, nb, gate = f["nw"], f["nb"], np.repeat(f["gate"], V, axis=0)
    h0 = q(P.norm(f["x"], nw[0], nb[0], False, EPS)[0])
    y1 = h0 @ q(f["w1"], True).T + f["b1"]
    y2 = q(y1) @ q(f["w2"], True).T
    t = P.block_norm_sum(y2, f["x"], nw[1], nb[1], f["res"], gate, False, EPS)
    z = q(P.norm(t, nw[2], nb[2], False, EPS)[0]) @ q(f["wz"], True).T
    rows, _, dz = P.distill(z, n["idx"], f["tl"], T, f["weight"])
    dh = q(dz) @ q(f["wz"], True)
    b = P.block_norm_backward(y2, t, None, dh, nw[1], nb[1], nw[2], f["res"], gate, False, EPS)
    return dict(t=t, z=z, rows=rows, loss=(rows * f["weight"]).sum(), dt=b["dx"], dy2=b["dy"], dy1=q(b["dy"]) @ q(f["w2"], True),
                dw2=q(b["dy"].T) @ q(y1.T).T, dpost_w=b["post_w"].sum(0), dpost_b=b["post_b"].sum(0), dpre_w=b["pre_w"].sum(0),
                dpre_b=b["pre_b"].sum(0), dres_scale=b["res_scale"].sum(0), dgate=b["gate"].reshape(N, V, C).sum(1))


def test_block_head_and_loss_forward_and_backward():
    s = Buffers(1)
    s.step()
    assert B.lamp_get_async_status() == 0
    ref = reference(s.np)
    for name, got in s.outputs().items():
        g, r = got.double().cpu().numpy().reshape(-1), np.asarray(ref[name], dtype=np.float64).reshape(-1)
        rel = np.linalg.norm(g - r) / np.linalg.norm(r)
        assert rel <= 0.05, (name, rel)


def test_step_in_a_graph_and_on_another_stream_gives_the_same_bits():
    s = Buffers(2)
    s.step()
    torch.cuda.synchronize()
    want = {n: v.clone() for n, v in s.outputs().items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.step()
    for _ in range(3):
        for v in s.outputs().values():
            v.zero_()
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(v, want[n]) for n, v in s.outputs().items())
    for v in s.outputs().values():
        v.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        s.step()
    torch.cuda.synchronize()
    assert all(torch.equal(v, want[n]) for n, v in s.outputs().items())
    assert B.lamp_get_async_status() == 0
