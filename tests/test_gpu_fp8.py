"""8-bit quantiser and matrix product on the GPU against the fp64 oracle.

Tolerances of the product.  Exact products of codes, summed in fp32: a term passes through at most 32 additions inside one
tensor-core instruction, 4 instructions per block, one scale product (2 roundings) and one addition per block, each off by
at most one unit of 2^-23 of the running magnitude (truncation counted as a full unit), so
    |y - ref| <= (40 + blocks) 2^-23 sum_k |a b| + 2^-23 |bias|,
plus half a step of the output type (bf16: 2^-8 relative)."""
import numpy as np
import pytest
import torch

from oracle import pointwise as P
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def bf16_values(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def operand(r, rows, k, tile, pad=0, scale_pad=0, spread=2.0):
    """Random codes and scales; what lies behind k and behind the scales is NaN and must never matter."""
    pitch = -(-k // 16) * 16 + pad
    codes = r.integers(0, 256, (rows, pitch)).astype(np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x21
    codes[:, k:] = 0x7F
    n = -(-rows // 128) if tile else rows
    scale = np.full((-(-k // 128), n + scale_pad), np.nan, dtype=np.float32)
    scale[:, :n] = np.exp(spread * r.standard_normal((scale.shape[0], n)))
    q, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scale).cuda()
    return B.fp8_operand(q, s, rows, k, tile), P.dequantize(codes[:, :k], scale[:, :n], tile)


def check(y, a, b, bias, out):
    ref = a @ b.T + (0 if bias is None else bias)
    mag = np.abs(a) @ np.abs(b).T
    blocks = -(-a.shape[1] // 128)
    tol = (40 + blocks) * 2.0 ** -23 * mag + 2.0 ** -23 * (0 if bias is None else np.abs(bias))
    if out is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    got = y.double().cpu().numpy()
    bad = np.abs(got - ref) > tol + 1e-37
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


SHAPES = [(1, 16, 16), (1, 200, 1), (1, 4096, 640), (2, 129, 257), (7, 1000, 4096), (17, 64, 100), (33, 300, 2048), (64, 128, 384), (64, 64, 128),
          (65, 129, 257), (128, 256, 2048), (130, 257, 1000), (300, 10, 512), (1000, 7, 33), (513, 48, 130), (640, 2000, 96), (200, 130, 5000)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_matches_oracle(m, n, k, out):
    r = np.random.default_rng(m * 7 + n + k)
    for i, (ta, tb, biased) in enumerate([(False, True, True), (False, False, False), (True, False, True)]):
        oa, a = operand(r, m, k, ta, pad=16 * i, scale_pad=i)
        ob, b = operand(r, n, k, tb, pad=16, scale_pad=3 * i)
        bias = r.standard_normal(n).astype(np.float32) if biased else None
        y = torch.full((1, 1, 1, m, n), float("nan"), dtype=out, device="cuda")
        B.lamp_gemm_fp8(oa, ob, y, None if bias is None else f32(bias))
        assert B.lamp_get_async_status() == 0
        check(y.view(m, n), a, b, bias, out)


@pytest.mark.parametrize("m,n,tile", [(2500, 2100, True), (2500, 2100, False), (4000, 300, True), (9600, 520, False), (5000, 130, True)])
def test_product_over_many_tiles(m, n, tile):
    # more tiles than SMs: the persistent walk, both scale kinds, an edge in both directions
    r = np.random.default_rng(5)
    oa, a = operand(r, m, 200, False)
    ob, b = operand(r, n, 200, tile)
    y = torch.empty((1, 1, 1, m, n), dtype=torch.float32, device="cuda")
    B.lamp_gemm_fp8(oa, ob, y)
    assert B.lamp_get_async_status() == 0
    check(y.view(m, n), a, b, None, torch.float32)


@pytest.mark.parametrize("m,n,k,ta,tb", [(500, 2000, 9000, False, False), (300, 1200, 5000, True, True), (1100, 1000, 2100, False, True), (260, 600, 7001, False, False),
                                         (1024, 1024, 2048, True, False)])
def test_long_reductions_are_shared_between_the_ctas_of_a_cluster(m, n, k, ta, tb):
    r = np.random.default_rng(6)
    oa, a = operand(r, m, k, ta)
    ob, b = operand(r, n, k, tb)
    for out in (torch.float32, torch.bfloat16):
        y = torch.empty((1, 1, 1, m, n), dtype=out, device="cuda")
        B.lamp_gemm_fp8(oa, ob, y)
        assert B.lamp_get_async_status() == 0
        check(y.view(m, n), a, b, None, out)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,pitch,off", [(5, 40, 64, 8), (200, 24, 61, 13), (150, 33, 40, 3), (300, 256, 288, 16), (300, 256, 272, 8)])
def test_product_into_a_channel_slice(m, n, pitch, off, out):
    r = np.random.default_rng(9)
    oa, a = operand(r, m, 300, False)
    ob, b = operand(r, n, 300, True)
    buf = torch.full((1, 1, 1, m, pitch), 7.0, dtype=out, device="cuda")
    B.lamp_gemm_fp8(oa, ob, B.tensor(buf, n, off))
    check(buf.view(m, pitch)[:, off:off + n], a, b, None, out)
    assert (buf[..., :off] == 7).all() and (buf[..., off + n:] == 7).all()


def test_nan_codes_and_extreme_scales_stay_in_their_rows():
    r = np.random.default_rng(11)
    for m, n in [(3, 200), (200, 140)]:
        oa, a = operand(r, m, 256, False)
        ob, b = operand(r, n, 256, True)
        oa.keep[0][1, 130] = 0x7F                            # one NaN code spoils its row and nothing else
        y = torch.empty((1, 1, 1, m, n), dtype=torch.float32, device="cuda")
        B.lamp_gemm_fp8(oa, ob, y)
        got = y.view(m, n).cpu().numpy()
        assert np.isnan(got[1]).all() and np.isfinite(np.delete(got, 1, 0)).all()
        oa.keep[0][1, 130] = 0
        # one block with a scale 2^40 above the others': the sum is that block's, to fp32
        oa.keep[1][1, :] *= 2.0 ** 40
        a2 = P.dequantize(oa.keep[0].cpu().numpy()[:, :256], oa.keep[1].cpu().numpy()[:, :m], False)
        B.lamp_gemm_fp8(oa, ob, y)
        check(y.view(m, n), a2, b, None, torch.float32)


def test_repeats_bit_for_bit_on_streams_and_in_graphs():
    r = np.random.default_rng(12)
    for m, n, k in [(1, 1024, 4096), (200, 300, 2000), (3000, 1500, 256)]:
        oa, _ = operand(r, m, k, False)
        ob, _ = operand(r, n, k, True)
        ys = [torch.full((1, 1, 1, m, n), float("nan"), device="cuda") for _ in range(4)]
        B.lamp_gemm_fp8(oa, ob, ys[0])
        side = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for st, y in zip(side, ys[1:3]):                     # two calls at once
            with torch.cuda.stream(st):
                B.lamp_gemm_fp8(oa, ob, y)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.lamp_gemm_fp8(oa, ob, ys[3])
        g.replay()
        ys[3].fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert B.lamp_get_async_status() == 0
        for y in ys[1:]:
            assert torch.equal(y, ys[0])


# --- quantiser: bit for bit ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,c", [(1, 8), (3, 128), (129, 136), (300, 264), (17, 1000), (128, 128), (1000, 24), (257, 512), (5, 12808), (700, 640)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("transpose,tile", [(False, False), (False, True), (True, False), (True, True)])
def test_quantise_matches_oracle(rows, c, dt, transpose, tile):
    r = np.random.default_rng(rows + c)
    x = r.standard_normal((rows, c)) * np.exp(3 * r.standard_normal((rows, 1)))
    x[r.random((rows, c)) < 0.1] = 0.0
    x = x.astype(np.float32)
    if rows > 100:
        x[5, 3], x[7, 2], x[9, 7] = np.nan, np.inf, -np.inf      # NaN codes; the block's scale comes from the others
        x[20:40] = 0                                             # zero blocks
        x[40] *= 1e-38                                           # below the smallest scale
        x[41] *= 1e30
    if dt is torch.bfloat16:
        x = bf16_values(x)
    m = x.T if transpose else x
    codes, scale = P.quantize(m, tile)
    R, K = m.shape
    pitch = -(-K // 16) * 16 + 16
    buf = torch.from_numpy(x).cuda().to(dt).view(1, 1, 1, rows, c)
    wide = torch.full((1, 1, 1, rows, c + 24), 3e4, dtype=dt, device="cuda")   # and from a channel slice
    wide[..., 16:16 + c] = buf
    for src in (buf, B.tensor(wide, c, 16)):
        q = torch.full((R, pitch), 0x55, dtype=torch.uint8, device="cuda")
        s = torch.full((scale.shape[0], scale.shape[1] + 5), -7.0, device="cuda")
        B.lamp_fp8_quantize(src, B.fp8_operand(q, s, R, K, tile), transpose)
        gq, gs = q.cpu().numpy(), s.cpu().numpy()
        np.testing.assert_array_equal(gs[:, :scale.shape[1]], scale)
        nan = np.isnan(P.e4m3_decode(codes))
        assert ((gq[:, :K][nan] & 0x7F) == 0x7F).all()
        np.testing.assert_array_equal(gq[:, :K][~nan], codes[~nan])
        assert (gq[:, K:] == 0x55).all() and (gs[:, scale.shape[1]:] == -7).all()   # nothing behind the operand is written


def test_quantised_layer_forward_and_both_gradients():
    """y = x W^T, dx = dy W, dW = dy^T x, each from the operand forms that the quantiser writes."""
    r = np.random.default_rng(21)
    R, K, N = 333, 264, 136
    x, w, dy = (bf16_values(r.standard_normal(s)) for s in ((R, K), (N, K), (R, N)))
    dev = lambda a: torch.from_numpy(a).cuda().to(torch.bfloat16).view(1, 1, 1, *a.shape)      # noqa: E731

    def quant(a, transpose, tile):
        m = a.T if transpose else a
        q = torch.zeros(m.shape[0], -(-m.shape[1] // 16) * 16, dtype=torch.uint8, device="cuda")
        s = torch.zeros(-(-m.shape[1] // 128), -(-m.shape[0] // 128) if tile else m.shape[0], device="cuda")
        o = B.fp8_operand(q, s, m.shape[0], m.shape[1], tile)
        B.lamp_fp8_quantize(dev(a), o, transpose)
        return o, P.dequantize(*P.quantize(m, tile), tile)

    for (a, ta, fa), (b, tb, fb), shape in [((x, False, False), (w, False, True), (R, N)), ((dy, False, False), (w, True, True), (R, K)),
                                            ((dy, True, False), (x, True, False), (N, K))]:
        oa, va = quant(a, ta, fa)
        ob, vb = quant(b, tb, fb)
        y = torch.empty((1, 1, 1, *shape), device="cuda")
        B.lamp_gemm_fp8(oa, ob, y)
        check(y.view(shape), va, vb, None, torch.float32)


def test_binding_refuses_what_a_pointer_would_not_show():
    r = np.random.default_rng(3)
    oa, _ = operand(r, 4, 64, False)
    ob, _ = operand(r, 8, 64, True)
    y = torch.empty((1, 1, 1, 4, 8), device="cuda")
    with pytest.raises(ValueError):
        B.lamp_gemm_fp8(oa, ob, y, torch.zeros(7, device="cuda"))
    with pytest.raises(ValueError):
        B.lamp_gemm_fp8(oa, ob, y, torch.zeros(8))
    with pytest.raises(ValueError):
        B.lamp_gemm_fp8(oa, ob, y.cpu())
    with pytest.raises(ValueError):
        B.fp8_operand(oa.keep[0], oa.keep[1], 5, 64)
    with pytest.raises(B.LampError):
        B.lamp_gemm_fp8(oa, ob, torch.empty((1, 1, 1, 4, 9), device="cuda"))
    # empty calls are no-ops
    e = torch.empty((1, 1, 1, 0, 8), device="cuda")
    B.lamp_gemm_fp8(B.fp8_operand(oa.keep[0], oa.keep[1], 0, 64), ob, e)
