"""The per-voxel operators where sizes are large: clusters that walk over many rows, weight gradients over 10^5 voxels and more, tensors of more
than 2^31 elements (offsets past 32 bits)."""
import numpy as np
import pytest
import torch

from paper_2006_12575_b200 import binding as B
from test_gpu_distill_range import check, listed

pytestmark = pytest.mark.gpu
FP8 = torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("c,dt", [(230000, torch.bfloat16), (120000, torch.float32)])
def test_clusters_of_eight_over_more_rows_than_clusters(c, dt):
    """At most two CTAs of such a cluster per SM, so at most 37 clusters on 148 SMs: each takes two or three rows."""
    rows, k = 85, 12
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    z = (2 * torch.randn(rows, c, device="cuda", generator=g)).to(dt)
    r = np.random.default_rng(1)
    check(z, listed(rows, c, k), (2 * r.standard_normal((rows, k))).astype(np.float32), 1.5)


def codes(g, rows, k):
    q = (torch.randn(rows, -(-k // 16) * 16, device="cuda", generator=g) * 60).clamp_(-448, 448).to(FP8)
    return q, torch.rand(-(-k // 128), rows, device="cuda", generator=g).mul_(0.02).add_(0.005)


def values(q, s, k, lo, hi):
    """Columns lo .. hi - 1 (multiples of 128) as 64-bit numbers."""
    return q[:, lo:hi].double() * s[lo // 128:-(-hi // 128)].double().t().repeat_interleave(128, 1)[:, :hi - lo]


@pytest.mark.parametrize("m,n,k", [(64, 64, 262144 + 40), (256, 256, 131072), (320, 96, 150001), (768, 768, 110000)])
def test_weight_gradient_over_many_voxels(m, n, k):
    """Tolerance of the product's tests: (40 + blocks) 2^-23 of the sum of magnitudes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m + k)
    (qa, sa), (qb, sb) = codes(g, m, k), codes(g, n, k)
    y = torch.full((1, 1, 1, m, n), float("nan"), device="cuda")
    B.lamp_gemm_fp8(B.fp8_operand(qa, sa, m, k), B.fp8_operand(qb, sb, n, k), y)
    assert B.lamp_get_async_status() == 0
    ref, mag = torch.zeros(m, n, dtype=torch.float64, device="cuda"), torch.zeros(m, n, dtype=torch.float64, device="cuda")
    for lo in range(0, k, 16384):
        a, b = (values(q, s, k, lo, min(k, lo + 16384)) for q, s in ((qa, sa), (qb, sb)))
        ref += a @ b.t()
        mag += a.abs() @ b.abs().t()
    assert ((y.view(m, n).double() - ref).abs() <= (40 + -(-k // 128)) * 2.0 ** -23 * mag).all()
    again = torch.empty_like(y)
    B.lamp_gemm_fp8(B.fp8_operand(qa, sa, m, k), B.fp8_operand(qb, sb, n, k), again)
    assert torch.equal(y, again)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tile", [False, True])
def test_quantise_transposed_over_many_voxels(dt, tile):
    rows, c = 300007, 136
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = (torch.randn(rows, c, device="cuda", generator=g) * torch.exp(torch.randn(1, c, device="cuda", generator=g))).to(dt)
    kb, rb = -(-rows // 128), -(-c // 128)
    q = torch.full((c, -(-rows // 16) * 16), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.zeros(kb, rb if tile else c, device="cuda")
    B.lamp_fp8_quantize(x.view(1, 1, 1, rows, c), B.fp8_operand(q, s, c, rows, tile), True)
    a = torch.zeros(rb * 128 if tile else c, kb * 128, device="cuda")
    a[:c, :rows] = x.float().t()
    amax = (a.view(rb, 128, kb, 128).abs().amax((1, 3)) if tile else a.view(c, kb, 128).abs().amax(2)).clamp_min(2.0 ** -100)
    assert torch.equal(s, (amax * torch.tensor(1.0 / 448.0, device="cuda")).t())
    inv = torch.full_like(amax, 448.0) / amax
    inv = (inv.repeat_interleave(128, 0)[:c] if tile else inv).repeat_interleave(128, 1)[:, :rows]
    assert torch.equal(q[:, :rows], (a[:c, :rows] * inv).to(FP8).view(torch.uint8)) and (q[:, rows:] == 0x55).all()


def test_product_of_more_than_2_31_outputs():
    m, n, k, tail = 70001, 32768, 128, 300                                 # 2.29e9 outputs, 4.6 GB
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    (qa, sa), (qb, sb) = codes(g, m, k), codes(g, n, k)
    y = torch.full((1, 1, 1, m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.lamp_gemm_fp8(B.fp8_operand(qa, sa, m, k), B.fp8_operand(qb, sb, n, k), y)
    assert B.lamp_get_async_status() == 0
    for rows in (slice(0, tail), slice(m - tail, m)):
        a, b = values(qa, sa, k, 0, k)[rows], values(qb, sb, k, 0, k)
        ref, mag = a @ b.t(), a.abs() @ b.abs().t()
        tol = 41 * 2.0 ** -23 * mag
        assert ((y.view(m, n)[rows].double() - ref).abs() <= tol + 2.0 ** -8 * (ref.abs() + tol)).all()
    assert not torch.isnan(y.view(-1)[:: 9973].float()).any()


@pytest.mark.parametrize("rows,c,k,tail", [(135000000, 16, 1, 1000), (2150000, 1000, 3, 1000), (44000, 50001, 8, 50)])
def test_distillation_of_more_than_2_31_logits(rows, c, k, tail):
    """The last rows against a call of their own, which may share a row between other numbers of CTAs and so add in another order.  Each of
    the two is within the bound of test_gpu_distill_range of the true value: with u = 2^-24, |z - max z| < 16, |log p| < 12, log c < 11 a
    log or a probability is within (112 + 55 + 80) u < 250 u, a loss of logs below 40 in sum within 40 (250 + 64) u + 3 * 250 u < 14000 u,
    and a gradient 0.5 (q - p) within 0.5 * 320 u (q + p) and half a step of bf16."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    z = torch.empty(1, 1, 1, rows, c, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    idx = torch.randint(0, c, (rows, k), device="cuda", generator=g, dtype=torch.int32)
    t, w = torch.randn(rows, k, device="cuda", generator=g), torch.full((rows,), 0.5, device="cuda")
    loss, own = torch.full((rows,), float("nan"), device="cuda"), torch.empty(tail, device="cuda")
    last = z[..., -tail:, :].clone()
    want = torch.empty_like(last)
    B.lamp_distill_topk_fwd_bwd(last, B.teacher_topk(idx[-tail:].clone(), t[-tail:].clone()), w[-tail:], own, None, want)
    B.lamp_distill_topk_fwd_bwd(z, B.teacher_topk(idx, t), w, loss, None, z)
    assert B.lamp_get_async_status() == 0
    assert not torch.isnan(loss).any() and ((loss[-tail:] - own).abs() <= 2 * 14000 * 2.0 ** -24).all()
    assert ((z[..., -tail:, :].double() - want.double()).abs() <= 2 * (2.0 ** -8 * want.double().abs() + 0.5 * 320 * 2.0 ** -24 * 2)).all()


def test_norms_of_more_than_2_31_elements():
    rows, c, tail = 4200000, 512, 500
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    new = lambda: torch.empty(1, 1, 1, rows, c, dtype=torch.bfloat16, device="cuda")                     # noqa: E731
    y, x, h = new().normal_(generator=g), new().normal_(generator=g), new()
    q, s = torch.zeros(rows, c, dtype=torch.uint8, device="cuda"), torch.zeros(4, rows, device="cuda")
    p = B.block_norm(pre_w=torch.rand(c, device="cuda", generator=g))
    end = lambda v: v[..., -tail:, :].clone()                                                            # noqa: E731
    yl, xl = end(y), end(x)
    ol, hl = torch.empty_like(xl), torch.empty_like(xl)
    ql, sl = torch.zeros(tail, c, dtype=torch.uint8, device="cuda"), torch.zeros(4, tail, device="cuda")
    B.lamp_block_norm_fwd(p, yl, xl, ol, hl, B.fp8_operand(ql, sl))
    B.lamp_block_norm_fwd(p, y, x, x, h, B.fp8_operand(q, s))
    assert torch.equal(end(x), ol) and torch.equal(end(h), hl) and torch.equal(q[-tail:], ql) and torch.equal(s[:, -tail:], sl)
    B.lamp_fp8_quantize(x, B.fp8_operand(q, s))
    B.lamp_fp8_quantize(ol, B.fp8_operand(ql, sl))
    assert torch.equal(q[-tail:], ql) and torch.equal(s[:, -tail:], sl)
    dxl, dyl = torch.empty_like(xl), torch.empty_like(xl)
    B.lamp_block_norm_bwd(p, yl, ol, xl, hl, dxl, dyl)
    x[..., -tail:, :] = xl
    t = new()
    t[..., -tail:, :] = ol
    t[..., :-tail, :] = 1.0
    B.lamp_block_norm_bwd(p, y, t, x, h, x, y)
    assert torch.equal(end(x), dxl) and torch.equal(end(y), dyl)
