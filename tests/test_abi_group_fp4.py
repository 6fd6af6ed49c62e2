"""Refusals of the group norm's, the clipping's and the 4-bit layers' entry points: decided on the host, nothing is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2006_12575_b200 import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40


def T(dt=B.LAMP_BF16, n=1, d=1, h=1, w=6, c=16, pitch=None, off=0, ptr=4096):
    return B.Tensor(ptr, dt, n, d, h, w, c, c if pitch is None else pitch, off)


def r(x):
    return C.byref(x) if x is not None else None


def gn(groups=4, act=2, slope=0.0, eps=1e-5, w=None, b=None):
    return B.GroupNorm(groups, act, slope, eps, w, b)


def fwd(p="p", x="x", z="z", stats=None, mr=4096, ws=4096, nb=BIG):
    d = {"p": gn(), "x": T(), "z": T()}
    g = lambda v: r(d[v]) if isinstance(v, str) else r(v)               # noqa: E731
    return B.lib().lamp_group_norm_act_fwd(g(p), g(x), stats, g(z), mr, ws, nb, None)


def bwd(p="p", dz="dz", x="x", dx="dx", mr=4096, dw=None, db=None, ws=4096, nb=BIG):
    d = {"p": gn(), "x": T(), "dz": T(), "dx": T()}
    g = lambda v: r(d[v]) if isinstance(v, str) else r(v)               # noqa: E731
    return B.lib().lamp_group_norm_act_bwd(g(p), g(dz), g(x), mr, g(dx), dw, db, ws, nb, None)


@pytest.mark.parametrize("call,other", [(fwd, "z"), (bwd, "dz"), (bwd, "dx")])
def test_group_norm_refusals(call, other):
    assert call(p=None) == INVALID and call(x=None) == INVALID and call(**{other: None}) == INVALID and call(mr=None) == INVALID
    for p in (gn(0), gn(-1), gn(5), gn(32), gn(act=4), gn(act=-1), gn(eps=-1.0), gn(eps=float("nan")), gn(slope=float("nan")), gn(slope=float("inf")),
              gn(w=4097), gn(b=4098)):
        assert call(p=p) == INVALID
    assert call(**{other: T(c=24)}) == INVALID and call(**{other: T(w=5)}) == INVALID and call(**{other: T(n=2, w=3)}) == INVALID
    assert call(**{other: T(B.LAMP_F32)}) == UNSUPPORTED                 # bf16 x, fp32 z or dz; dx of another type than x
    for t in (T(c=12), T(pitch=18), T(pitch=32, off=4)):
        assert call(x=t) == UNSUPPORTED
    f = T(B.LAMP_F32, c=12)
    assert call(p=gn(4), x=f, **{other: f}) == UNSUPPORTED
    assert call(x=T(ptr=4104)) == INVALID and call(mr=4100) == INVALID
    assert call(ws=None) == WORKSPACE and call(ws=4104) == WORKSPACE
    need = B.lib().lamp_group_norm_workspace_bytes(r(gn()), r(T()))
    assert need > 0 and call(nb=need - 1) == WORKSPACE
    huge = T(c=65544, w=1)
    assert call(p=gn(1), x=huge, **({"z": huge} if call is fwd else {"dz": huge, "dx": huge})) == UNSUPPORTED


def test_group_norm_more_refusals():
    assert fwd(stats=4104, ws=None) == INVALID                           # fp64 pairs
    assert bwd(dw=4097) == INVALID and bwd(db=4098) == INVALID
    e = T(w=0)
    assert fwd(x=e, z=e, ws=None) == OK and bwd(x=e, dz=e, dx=e, ws=None) == OK
    L = B.lib()
    assert L.lamp_group_norm_workspace_bytes(None, r(T())) == 0 and L.lamp_group_norm_workspace_bytes(r(gn()), None) == 0
    assert L.lamp_group_norm_workspace_bytes(r(gn(5)), r(T())) == 0 and L.lamp_group_norm_workspace_bytes(r(gn()), r(T(w=0))) == 0


def G(n=4, dt=B.LAMP_F32, g=4096, out=8192):
    return B.Grad(g, out, n, dt)


def clip(*grads, count=None, max_norm=1.0, norm=4096, factor=4096, ws=4096, nb=BIG, scale=True):
    a = (B.Grad * max(1, len(grads)))(*grads)
    f = B.lib().lamp_grad_clip if scale else B.lib().lamp_grad_norm
    return f(a, len(grads) if count is None else count, max_norm, norm, factor, ws, nb, None)


def test_clip_refusals():
    for scale in (True, False):
        assert clip(G(), scale=scale, norm=None) == INVALID and clip(G(), scale=scale, norm=4098) == INVALID
        assert clip(G(), scale=scale, max_norm=-1.0) == INVALID and clip(G(), scale=scale, max_norm=float("nan")) == INVALID
        assert clip(G(), scale=scale, count=-1) == INVALID and clip(G(), scale=scale, count=(1 << 20) + 1) == UNSUPPORTED
        assert clip(G(n=-1), scale=scale) == INVALID and clip(G(n=(1 << 40) + 1), scale=scale) == UNSUPPORTED
        assert clip(*[G(n=1 << 40) for _ in range(5)], scale=scale) == UNSUPPORTED
        assert clip(G(dt=2), scale=scale) == UNSUPPORTED
        assert clip(G(g=None), scale=scale) == INVALID and clip(G(g=4098), scale=scale) == INVALID and clip(G(dt=B.LAMP_BF16, g=4097), scale=scale) == INVALID
        need = B.lib().lamp_grad_norm_workspace_bytes((B.Grad * 1)(G()), 1)
        assert need > 0 and clip(G(), scale=scale, nb=need - 1) == WORKSPACE
        assert clip(G(), scale=scale, ws=None) == WORKSPACE and clip(G(), scale=scale, ws=4104) == WORKSPACE
    assert clip(G(), factor=None) == INVALID and clip(G(), factor=4098, scale=False) == INVALID
    assert clip(G(out=None)) == INVALID and clip(G(out=8194)) == INVALID
    L = B.lib()
    assert L.lamp_grad_clip(None, 1, 1.0, 4096, 4096, 4096, BIG, None) == INVALID
    assert L.lamp_grad_norm_workspace_bytes(None, 1) == 0 and L.lamp_grad_norm_workspace_bytes(None, 0) > 0
    many = (B.Grad * 2500)(*[G() for _ in range(2500)])
    assert L.lamp_grad_norm_workspace_bytes(many, 2500) >= 3 * L.lamp_grad_norm_workspace_bytes(many, 1)


def test_scaled_update_refusals():
    f = lambda n=8, g=4096, s=4096, w=4096, v=4096, p=None, lr=0.1, a=0.9, e=0.0: B.lib().lamp_rmsprop_step_scaled(n, g, s, w, v, p, lr, a, e, None)   # noqa: E731
    assert f(n=-1) == INVALID and f(n=0) == OK
    assert f(g=None) == INVALID and f(s=None) == INVALID and f(w=None) == INVALID and f(v=None) == INVALID
    assert f(s=4098) == INVALID and f(g=4098) == INVALID and f(p=4097) == INVALID
    assert f(lr=-1.0) == INVALID and f(a=1.5) == INVALID and f(e=-1.0) == INVALID


def F(rows=6, k=16, pitch=None, block=32, q=4096, s=4096, ts=None):
    return B.Fp4Operand(q, -(-(-(-k // 2)) // 16) * 16 if pitch is None else pitch, s, ts, rows, k, block)


def gemm(a=None, b=None, y=None, bias=None):
    return B.lib().lamp_gemm_fp4(r(a or F(6, 32)), r(b or F(8, 32)), bias, r(y or T(w=6, c=8)), None)


def test_fp4_gemm_refusals():
    assert gemm(a=F(6, 48)) == INVALID and gemm(a=F(6, 32, block=16)) == INVALID                 # k, block differ
    assert gemm(a=F(7, 32)) == INVALID and gemm(b=F(9, 32)) == INVALID
    assert gemm(a=F(6, 32, pitch=8)) == INVALID and gemm(a=F(6, 33, pitch=16), b=F(8, 33)) == INVALID and gemm(a=F(6, 32, pitch=24)) == INVALID
    assert gemm(a=F(6, 32, q=4104)) == INVALID and gemm(a=F(6, 32, s=4100)) == INVALID and gemm(a=F(6, 32, q=None)) == INVALID
    assert gemm(a=F(6, 32, s=None)) == INVALID and gemm(a=F(6, 32, block=8)) == INVALID and gemm(a=F(-1, 32)) == INVALID
    assert gemm(a=F(6, 32, ts=4096)) == INVALID                                                  # no tensor scale with blocks of 32
    assert gemm(a=F(6, 32, block=16, ts=4098), b=F(8, 32, block=16)) == INVALID
    assert gemm(a=F(6, 0), b=F(8, 0)) == INVALID and gemm(bias=4097) == INVALID
    assert gemm(y=B.Tensor(4096, 2, 1, 1, 1, 6, 8, 8, 0)) == UNSUPPORTED and gemm(a=F(2 ** 31, 32)) == UNSUPPORTED
    L = B.lib()
    assert L.lamp_gemm_fp4(None, r(F(8, 32)), None, r(T(c=8)), None) == INVALID
    assert L.lamp_gemm_fp4(r(F(6, 32)), r(F(8, 32)), None, None, None) == INVALID
    assert gemm(a=F(0, 32), y=T(w=0, c=8)) == OK


@pytest.mark.parametrize("back", [False, True])
def test_fp4_conversion_refusals(back):
    def q(x, t, o):
        return B.lib().lamp_fp4_dequantize(r(o), t, r(x), None) if back else B.lib().lamp_fp4_quantize(r(x), t, r(o), None)
    assert q(None, 0, F()) == INVALID and q(T(), 0, None) == INVALID and q(T(), 2, F()) == INVALID
    assert q(T(), 0, F(6, 17)) == INVALID and q(T(), 0, F(5, 16)) == INVALID and q(T(), 1, F(6, 16)) == INVALID
    for dt in (B.LAMP_BF16, B.LAMP_F32):
        assert q(T(dt, c=12), 0, F(6, 12)) == UNSUPPORTED and q(T(dt, pitch=18), 0, F()) == UNSUPPORTED and q(T(dt, pitch=32, off=4), 0, F()) == UNSUPPORTED
    assert q(T(ptr=4100), 0, F()) == INVALID and q(T(), 0, F(block=64)) == INVALID and q(T(), 0, F(ts=4096)) == INVALID
    assert q(T(w=0), 0, F(0, 16)) == OK and q(T(w=0), 1, F(16, 0)) == OK


def test_scale_bytes():
    f = B.lamp_fp4_scale_bytes
    assert f(1, 1, 32) == 512 and f(128, 128, 32) == 512 and f(129, 129, 32) == 2048 and f(128, 65, 16) == 1024 and f(0, 5, 16) == 0
    assert f(-1, 5, 16) == 0 and f(5, 5, 8) == 0 and f(2 ** 31, 5, 16) == 0


def test_binding_checks_need_no_launch():
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)            # noqa: E731
    u8 = torch.uint8
    with pytest.raises(ValueError):
        B.fp4_operand(z(4, 16, dt=u8), z(512, dt=u8))                     # not on a GPU
    with pytest.raises(ValueError):
        B.group_norm(4, act="swish")
    with pytest.raises(ValueError):
        B.group_norm(4, z(16), z(8))
    assert B.group_norm(4, act="leaky_relu", slope=0.01).act == 1
    with pytest.raises(ValueError):
        B.grad_list([z(4)])                                               # not on a GPU
    with pytest.raises(ValueError):
        B.grad_list([z(4)], [])
    assert B.grad_list([]).count == 0
