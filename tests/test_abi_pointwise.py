"""Refusals of the per-voxel operators' entry points: decided on the host, nothing is launched (no GPU needed)."""
import ctypes as C

import pytest

from paper_2006_12575_b200 import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


def T(dt=B.LAMP_BF16, n=1, d=1, h=1, w=6, c=16, pitch=None, off=0, ptr=4096):
    return B.Tensor(ptr, dt, n, d, h, w, c, c if pitch is None else pitch, off)


def F(rows=6, k=16, pitch=None, sp=None, tile=0, q=4096, s=4096):
    return B.Fp8Operand(q, -(-k // 16) * 16 if pitch is None else pitch, s, rows if sp is None else sp, rows, k, tile)


def r(x):
    return C.byref(x) if x is not None else None


def gemm(a=None, b=None, y=None, bias=None):
    return B.lib().lamp_gemm_fp8(r(a or F(6, 32)), r(b or F(8, 32)), bias, r(y or T(w=6, c=8)), None)


def test_gemm_refusals():
    assert gemm(a=F(6, 48)) == INVALID                                  # k differs
    assert gemm(a=F(7, 32)) == INVALID and gemm(b=F(9, 32)) == INVALID  # rows differ from y's voxels / channels
    assert gemm(a=F(6, 32, pitch=24)) == INVALID                        # pitch below k
    assert gemm(a=F(6, 32, pitch=40)) == INVALID                        # not a multiple of 16
    assert gemm(a=F(6, 32, q=4104)) == INVALID and gemm(a=F(6, 32, s=4097)) == INVALID
    assert gemm(a=F(6, 32, q=0)) == INVALID and gemm(a=F(6, 32, s=0)) == INVALID
    assert gemm(a=F(6, 32, sp=5)) == INVALID
    assert gemm(a=F(6, 32, tile=2)) == INVALID and gemm(a=F(-1, 32)) == INVALID
    assert gemm(bias=4097) == INVALID
    assert gemm(a=F(6, 0), b=F(8, 0)) == INVALID                        # nothing to sum
    assert gemm(y=B.Tensor(4096, 2, 1, 1, 1, 6, 8, 8, 0)) == UNSUPPORTED
    assert gemm(a=F(2 ** 31, 32)) == UNSUPPORTED
    L = B.lib()
    assert L.lamp_gemm_fp8(None, r(F(8, 32)), None, r(T(c=8)), None) == INVALID
    assert L.lamp_gemm_fp8(r(F(6, 32)), r(F(8, 32)), None, None, None) == INVALID
    assert gemm(a=F(0, 32), y=T(w=0, c=8)) == OK                        # no rows: nothing to do


def test_quantize_refusals():
    q = lambda x, t, o: B.lib().lamp_fp8_quantize(r(x), t, r(o), None)  # noqa: E731
    assert q(None, 0, F()) == INVALID and q(T(), 0, None) == INVALID
    assert q(T(), 2, F()) == INVALID
    assert q(T(), 0, F(6, 17)) == INVALID and q(T(), 0, F(5, 16)) == INVALID
    assert q(T(), 1, F(6, 16)) == INVALID                               # transposed: 16 rows of 6
    assert q(T(c=12), 0, F(6, 12)) == UNSUPPORTED                       # c not a multiple of 8
    assert q(T(B.LAMP_F32, c=12), 0, F(6, 12)) == UNSUPPORTED
    assert q(T(pitch=18), 0, F()) == UNSUPPORTED and q(T(pitch=32, off=4), 0, F()) == UNSUPPORTED
    assert q(T(ptr=4100), 0, F()) == INVALID
    assert q(T(w=0), 0, F(0, 16)) == OK


def norm(p=None, y="y", x="x", out="o", h="h", f=None):
    d = {"y": T(), "x": T(), "o": T(), "h": T()}
    g = lambda v: r(d[v]) if isinstance(v, str) else r(v)               # noqa: E731
    return B.lib().lamp_block_norm_fwd(r(p if p is not None else B.BlockNorm(0, 1e-5)), g(y), g(x), g(out), g(h), r(f), None)


def test_block_norm_forward_refusals():
    L = B.lib()
    assert L.lamp_block_norm_fwd(None, r(T()), r(T()), r(T()), r(T()), None, None) == INVALID
    assert norm(x=None) == INVALID and norm(out=None) == INVALID and norm(y=None) == INVALID
    assert norm(y=None, out=None, h=None) == INVALID                    # nothing asked for
    assert norm(p=B.BlockNorm(2, 1e-5)) == INVALID and norm(p=B.BlockNorm(0, -1.0)) == INVALID and norm(p=B.BlockNorm(0, float("nan"))) == INVALID
    assert norm(y=T(c=24)) == INVALID and norm(out=T(w=5)) == INVALID and norm(h=T(n=2, w=3)) == INVALID
    assert norm(y=T(B.LAMP_F32)) == UNSUPPORTED                         # branch tensors of two types
    assert norm(y=T(B.LAMP_F32), h=T(B.LAMP_F32)) == UNSUPPORTED        # bf16 stream, fp32 branch
    assert norm(out=T(B.LAMP_F32)) == UNSUPPORTED
    big = T(c=8200)
    assert norm(y=big, x=big, out=big, h=big) == UNSUPPORTED
    odd = T(B.LAMP_F32, c=12)
    assert norm(y=odd, x=odd, out=odd, h=odd) == UNSUPPORTED
    assert norm(h=None, f=F(6, 17)) == INVALID and norm(h=None, f=F(6, 16, tile=1)) == INVALID
    p = B.BlockNorm(0, 1e-5)
    lg = T()
    p.gate, p.gate_logits = 4096, C.pointer(lg)
    assert norm(p=p) == INVALID                                         # two gates
    p = B.BlockNorm(0, 1e-5)
    p.post_w = 4098
    assert norm(p=p) == INVALID
    p = B.BlockNorm(0, 1e-5)
    p.res_scale = 4096
    assert norm(p=p, y=None, out=None) == INVALID                       # a residual scale without a post-norm
    e = T(w=0)
    assert norm(y=e, x=e, out=e, h=e) == OK


def test_block_norm_backward_refusals():
    L = B.lib()
    g = B.BlockNormGrads()

    def bwd(p=None, y=None, t=None, do=None, dh=None, dx=None, dy=None, dl=None, grads=g, ws=None, nb=0, drop=()):
        a = dict(y=y or T(), t=t or T(), do=do or T(), dh=dh or T(), dx=dx or T(), dy=dy or T(), dl=dl)
        for n in drop:
            a[n] = None
        return L.lamp_block_norm_bwd(r(p or B.BlockNorm(0, 1e-5)), r(a["y"]), r(a["t"]), r(a["do"]), r(a["dh"]), r(a["dx"]), r(a["dy"]),
                                     r(a["dl"]), r(grads), ws, nb, None)
    assert bwd(drop=("t",)) == INVALID and bwd(drop=("dx",)) == INVALID and bwd(drop=("do", "dh")) == INVALID
    assert bwd(drop=("y",)) == INVALID and bwd(drop=("dy",)) == INVALID
    assert bwd(drop=("y", "dy", "dh")) == INVALID                       # no norm at all
    assert bwd(dl=T()) == INVALID                                       # no logits
    assert bwd(do=T(c=24)) == INVALID and bwd(dx=T(B.LAMP_F32)) == UNSUPPORTED
    assert bwd(y=T(B.LAMP_F32)) == UNSUPPORTED
    want = B.BlockNormGrads()
    want.pre_w = 4096
    need = L.lamp_block_norm_bwd_workspace_bytes(r(T()), r(B.BlockNorm(0, 1e-5)))
    assert need > 0 and need % (16 * 4 * 4) == 0
    assert bwd(grads=want) == WORKSPACE and bwd(grads=want, ws=4096, nb=need - 1) == WORKSPACE and bwd(grads=want, ws=4104, nb=need) == WORKSPACE
    want.gate = 4096
    assert bwd(grads=want, ws=4096, nb=need) == INVALID                 # a gate's gradient without a gate
    assert L.lamp_block_norm_bwd_workspace_bytes(None, r(B.BlockNorm(0, 1e-5))) == 0
    assert L.lamp_block_norm_bwd_workspace_bytes(r(T(c=12)), r(B.BlockNorm(0, 1e-5))) == 0


def test_distill_refusals():
    L = B.lib()

    def K(k=4, temp=1.0, idx=4096, t=4096, lse=None):
        return B.TeacherTopk(idx, t, lse, k, temp)

    def fwd(z=None, t=None, w=None, rows=4096, lse=None, loss=None, ws=None, nb=0):
        return L.lamp_distill_topk_fwd(r(z or T()), r(t or K()), w, rows, lse, loss, ws, nb, None)
    assert L.lamp_distill_topk_fwd(None, r(K()), None, 4096, None, None, None, 0, None) == INVALID
    assert L.lamp_distill_topk_fwd(r(T()), None, None, 4096, None, None, None, 0, None) == INVALID
    assert fwd(t=K(k=0)) == INVALID and fwd(t=K(k=1025)) == UNSUPPORTED
    for temp in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(t=K(temp=temp)) == INVALID
    assert fwd(t=K(idx=None)) == INVALID and fwd(t=K(t=None)) == INVALID and fwd(t=K(idx=4098)) == INVALID
    assert fwd(rows=None) == INVALID                                    # nothing asked for
    assert fwd(w=4098) == INVALID and fwd(rows=4098) == INVALID
    need = L.lamp_distill_topk_workspace_bytes(r(T()))
    assert need > 0 and L.lamp_distill_topk_workspace_bytes(None) == 0
    assert fwd(loss=4096) == WORKSPACE and fwd(loss=4096, ws=4096, nb=need - 1) == WORKSPACE and fwd(loss=4096, ws=4104, nb=need) == WORKSPACE
    bwd = lambda z, dz, lse=4096: L.lamp_distill_topk_bwd(r(z), r(K()), None, lse, r(dz), None)      # noqa: E731
    assert bwd(T(), None) == INVALID and bwd(T(), T(c=24)) == INVALID and bwd(T(), T(B.LAMP_F32)) == UNSUPPORTED
    assert bwd(T(), T(), None) == INVALID
    assert L.lamp_distill_topk_fwd_bwd(r(T()), r(K()), None, None, None, None, None, 0, None) == INVALID
    e = T(w=0)
    assert bwd(e, e) == OK


def test_binding_checks_need_no_launch():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        B.fp8_operand(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(1, 4))          # not on a GPU
    with pytest.raises(ValueError):
        B.teacher_topk(torch.zeros(4, dtype=torch.int32), torch.zeros(4))
