"""4-bit quantiser, its inverse and the 4-bit matrix product on the GPU against the oracle.

The quantiser is compared bit for bit: the oracle does every fp32 operation of the definition.
Tolerance of the product.  A product of two codes and two scales is exact in fp32 (at most 12 significant bits).  Summed in fp32, a term
passes through at most 64 additions inside one tensor-core instruction, k / 64 instructions and, where CTAs share the k axis, 8 more additions,
each off by at most one unit of 2^-23 of the running magnitude (truncation counted as a full unit); ga * gb, its product with the sum and
the bias take three roundings:
    |y - ref| <= (76 + k / 64) 2^-23 sum_k |a b| + 2^-23 |bias|,
plus half a step of the output type (bf16: 2^-8 relative)."""
import numpy as np
import pytest
import torch

from oracle import fp4 as Q
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def operand(r, rows, k, block, g=None, pad=0):
    """Random codes and scales.  What lies behind ceil(k / 2) bytes and in the scales of rows that do not exist must never matter: any byte, NaN
    scales among them."""
    pitch = -(-(-(-k // 2)) // 16) * 16 + pad
    codes = r.integers(0, 16, (rows, k)).astype(np.uint8)
    q = r.integers(0, 256, (rows, pitch)).astype(np.uint8)
    held = Q.pack(codes, pitch)
    q[:, :-(-k // 2)] = held[:, :-(-k // 2)]
    kb = -(-k // block)
    scales = r.integers(117, 133, (rows, kb)).astype(np.uint8) if block == 32 else r.integers(0x18, 0x58, (rows, kb)).astype(np.uint8)
    sb = np.full(Q.scale_bytes(rows, k, block), 255 if block == 32 else 127, np.uint8)
    rows128, kb4 = -(-rows // 128) * 128, -(-kb // 4) * 4
    places = Q.scale_places(rows128, kb4)
    sb[places[:rows]] = 0                                            # blocks behind the last of a row: 0, as the quantiser leaves them
    sb[places[:rows, :kb]] = scales
    tg = f32([g]) if g is not None else None
    op = B.fp4_operand(u8(q), u8(sb), rows, k, block, tg)
    return op, Q.dequantize(codes, scales, block, 1.0) * (1.0 if g is None else float(np.float32(g)))


def check(y, a, b, bias, out):
    ref = a @ b.T + (0 if bias is None else bias)
    tol = (76 + a.shape[1] // 64) * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T) + 2.0 ** -23 * (0 if bias is None else np.abs(bias))
    if out is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= tol + 1e-37)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


SHAPES = [(1, 16, 16), (1, 200, 1), (1, 4096, 640), (2, 129, 257), (7, 1000, 4096), (17, 64, 100), (33, 300, 2048), (64, 128, 384), (64, 64, 128),
          (65, 129, 257), (128, 256, 2048), (130, 257, 1000), (300, 10, 512), (1000, 7, 33), (513, 48, 130), (640, 2000, 96), (200, 130, 5000),
          (100, 100, 31), (300, 40, 65)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("block", [32, 16])
def test_product_matches_oracle(m, n, k, block):
    r = np.random.default_rng(m * 7 + n + k)
    for i, (out, biased) in enumerate([(torch.float32, True), (torch.bfloat16, False)]):
        oa, a = operand(r, m, k, block, 0.37 if block == 16 else None, 16 * i)
        ob, b = operand(r, n, k, block, 3.0 if block == 16 and i == 0 else None, 32 * i)
        bias = r.standard_normal(n).astype(np.float32) * 50 if biased else None
        y = torch.full((1, 1, 1, m, n), float("nan"), dtype=out, device="cuda")
        B.lamp_gemm_fp4(oa, ob, y, f32(bias) if biased else None)
        assert B.lamp_get_async_status() == 0
        check(y.view(m, n), a, b, bias, out)


# tiles of CTA pairs: 256 x 256, 256 x 128, with rows and columns that leave parts of a pair empty
@pytest.mark.parametrize("m,n,k", [(2300, 2100, 300), (5000, 512, 544), (19000, 128, 257), (10000, 200, 700), (2560, 2048, 2048)])
@pytest.mark.parametrize("block", [32, 16])
def test_product_in_pairs_matches_oracle(m, n, k, block):
    r = np.random.default_rng(m + n + k)
    for out in (torch.bfloat16, torch.float32):
        oa, a = operand(r, m, k, block, 0.37 if block == 16 else None, 16)
        ob, b = operand(r, n, k, block)
        bias = r.standard_normal(n).astype(np.float32) * 50
        y = torch.full((1, 1, 1, m, n), float("nan"), dtype=out, device="cuda")
        B.lamp_gemm_fp4(oa, ob, y, f32(bias))
        assert B.lamp_get_async_status() == 0
        check(y.view(m, n), a, b, bias, out)
        again = torch.empty_like(y)
        B.lamp_gemm_fp4(oa, ob, again, f32(bias))
        assert torch.equal(y, again)


@pytest.mark.parametrize("m,n", [(130, 40), (7, 300), (2500, 1300)])
def test_product_into_a_channel_slice(m, n):
    r = np.random.default_rng(m)
    oa, a = operand(r, m, 192, 32)
    ob, b = operand(r, n, 192, 32)
    for out, off in ((torch.bfloat16, 3), (torch.float32, 1), (torch.bfloat16, 16)):
        y = torch.full((1, 1, 1, m, n + 29), 7.0, dtype=out, device="cuda")
        B.lamp_gemm_fp4(oa, ob, B.tensor(y, n, off))
        v = y.view(m, -1)
        check(v[:, off:off + n], a, b, None, out)
        assert (v[:, :off] == 7).all() and (v[:, off + n:] == 7).all()


@pytest.mark.parametrize("block", [32, 16])
def test_nan_scale_reaches_only_its_row(block):
    r = np.random.default_rng(1)
    oa, a = operand(r, 70, 300, block)
    ob, b = operand(r, 90, 300, block)
    kb = -(-300 // block)
    oa.keep[1][int(Q.scale_places(70, kb)[5, 2])] = 255 if block == 32 else 127
    y = torch.empty(1, 1, 1, 70, 90, device="cuda")
    B.lamp_gemm_fp4(oa, ob, y)
    v = y.view(70, 90)
    assert v[5].isnan().all()
    keep = [i for i in range(70) if i != 5]
    check(v[keep], a[keep], b, None, torch.float32)


def values(r, rows, c, dt):
    x = r.standard_normal((rows, c)) * np.exp(1.5 * r.standard_normal((1, c)))
    x[::7] = np.maximum(x[::7], 0)
    x[rows // 2] = 0
    x[rows // 3, :8] = [1e-30, -1e-38, 3e38, -3e38, 1e-42, 6, 0.75, -0.0]
    x = x.astype(np.float32)
    return x if dt is torch.float32 else torch.from_numpy(x).to(torch.bfloat16).float().numpy()


@pytest.mark.parametrize("rows,c", [(1, 8), (3, 128), (130, 136), (257, 264), (1000, 40), (300, 32), (33, 1024), (700, 520)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("transpose", [False, True])
def test_quantiser_bit_for_bit_and_back(rows, c, dt, block, transpose):
    r = np.random.default_rng(rows + c)
    x = values(r, rows, c, dt)
    g = None if block == 32 else np.float32(0.7)
    wide = torch.full((1, 1, 1, rows, c + 24), 9.0, dtype=dt, device="cuda")
    wide[0, 0, 0, :, 8:8 + c] = torch.from_numpy(x).cuda().to(dt)
    rr, k = (c, rows) if transpose else (rows, c)
    pitch = -(-(-(-k // 2)) // 16) * 16 + 16
    q, s = torch.full((rr, pitch), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((Q.scale_bytes(rr, k, block) + 16,), 0xEE, dtype=torch.uint8, device="cuda")
    op = B.fp4_operand(q, s, rr, k, block, None if g is None else f32([g]))
    B.lamp_fp4_quantize(B.tensor(wide, c, 8), op, transpose)
    codes, scales = Q.quantize(x.T if transpose else x, block, 1.0 if g is None else g)
    got = q.cpu().numpy()
    nb = -(-k // 2)
    np.testing.assert_array_equal(got[:, :nb], Q.pack(codes, pitch)[:, :nb])          # an odd k leaves 0 in the last half byte
    assert (got[:, nb:] == 0xA5).all()
    sb = np.zeros(Q.scale_bytes(rr, k, block), np.uint8)                              # 0 where a tile of scales has no row or block
    sb[Q.scale_places(rr, scales.shape[1])] = scales
    np.testing.assert_array_equal(s.cpu().numpy()[:-16], sb)
    assert (s[-16:] == 0xEE).all()
    ref = Q.dequantize(codes, scales, block, 1.0 if g is None else g).astype(np.float32)
    y = torch.full((1, 1, 1, rows, c + 24), 9.0, dtype=dt, device="cuda")
    B.lamp_fp4_dequantize(op, B.tensor(y, c, 8), transpose)
    np.testing.assert_array_equal(y[0, 0, 0, :, 8:8 + c].float().cpu().numpy(), torch.from_numpy(ref.T.copy() if transpose else ref).to(dt).float().numpy())
    assert (y[..., :8] == 9).all() and (y[..., 8 + c:] == 9).all()


@pytest.mark.parametrize("block", [32, 16])
def test_ties_and_borders(block):
    """Every code's borders and their neighbours under scales of full precision; blocks of 16: ties hold where x / (scale g) is exact."""
    steps = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], np.float32)
    near = np.concatenate([steps, np.nextafter(steps, np.float32(0)), np.nextafter(steps, np.float32(9))])
    rows = []
    for scale in (1.0, 2.0 ** -20, 2.0 ** 60) if block == 32 else [float(v) for v in Q.E4M3[8:126]]:
        v = (near * np.float32(scale)).astype(np.float32)
        for i in range(0, 24, 12):
            row = np.zeros(block, np.float32)
            row[:12], row[12], row[13] = v[i:i + 12], 6 * scale, -2.5 * scale
            rows.append(row)
    x = np.array(rows)
    q, s = torch.zeros(len(x), 16, dtype=torch.uint8, device="cuda"), torch.zeros(Q.scale_bytes(len(x), block, block), dtype=torch.uint8, device="cuda")
    op = B.fp4_operand(q, s, len(x), block, block)
    B.lamp_fp4_quantize(f32(x).view(1, 1, 1, len(x), block), op)
    codes, _ = Q.quantize(x, block)
    np.testing.assert_array_equal(q.cpu().numpy(), Q.pack(codes, 16))


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_blocks_that_are_not_finite(block, transpose, dt):
    r = np.random.default_rng(0)
    x = r.standard_normal((96, 96)).astype(np.float32)
    x = torch.from_numpy(x).to(dt).float().numpy()
    x[5, 40], x[33, 33], x[70, 2] = np.nan, np.inf, -np.inf
    q, s = torch.zeros(96, 48, dtype=torch.uint8, device="cuda"), torch.zeros(Q.scale_bytes(96, 96, block), dtype=torch.uint8, device="cuda")
    op = B.fp4_operand(q, s, 96, 96, block)
    B.lamp_fp4_quantize(f32(x).to(dt).view(1, 1, 1, 96, 96), op, transpose)
    codes, scales = Q.quantize(x.T if transpose else x, block)
    np.testing.assert_array_equal(q.cpu().numpy(), Q.pack(codes, 48))
    np.testing.assert_array_equal(s.cpu().numpy()[Q.scale_places(96, scales.shape[1])], scales)
    y = torch.empty(1, 1, 1, 96, 96, dtype=dt, device="cuda")
    B.lamp_fp4_dequantize(op, y, transpose)
    v = y.view(96, 96)
    assert v.isnan().sum() == 3 * block and v[5, 40].isnan() and v[33, 33].isnan() and v[70, 2].isnan()


@pytest.mark.parametrize("block", [32, 16])
def test_on_a_side_stream_and_in_a_graph(block):
    r = np.random.default_rng(4)
    x, w = r.standard_normal((300, 264)).astype(np.float32), r.standard_normal((72, 264)).astype(np.float32)
    tx, tw = f32(x).view(1, 1, 1, 300, 264), f32(w).view(1, 1, 1, 72, 264)
    ops = [B.fp4_operand(torch.zeros(n, 144, dtype=torch.uint8, device="cuda"), torch.zeros(Q.scale_bytes(n, 264, block), dtype=torch.uint8, device="cuda"), n, 264, block)
           for n in (300, 72)]
    y = torch.zeros(1, 1, 1, 300, 72, device="cuda")

    def run():
        B.lamp_fp4_quantize(tx, ops[0])
        B.lamp_fp4_quantize(tw, ops[1])
        B.lamp_gemm_fp4(ops[0], ops[1], y)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        run()
    st.synchronize()
    check(y.view(300, 72), Q.dequantize(*Q.quantize(x, block), block), Q.dequantize(*Q.quantize(w, block), block), None, torch.float32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    x2 = r.standard_normal((300, 264)).astype(np.float32)
    tx.copy_(f32(x2).view_as(tx))
    g.replay()
    torch.cuda.synchronize()
    check(y.view(300, 72), Q.dequantize(*Q.quantize(x2, block), block), Q.dequantize(*Q.quantize(w, block), block), None, torch.float32)
