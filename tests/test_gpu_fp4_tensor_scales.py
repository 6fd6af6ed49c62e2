"""4-bit product whose tensor scales are no ordinary numbers: ga * gb beyond fp32's range, or below its normal numbers, while the results are not.

Tolerance: that of the product's other tests, (76 + k / 64) 2^-23 sum |a b| - the two factors one after the other round twice, as their
product and its product with the sum do - and half a step of the output type; below the normal range half of its smallest step, twice."""
import numpy as np
import pytest
import torch

from oracle import fp4 as Q
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
# rows of a, rows of b, k: b on the lanes, one CTA per tile, the k axis shared, pairs of 256 and 128 columns
SHAPES = [(3, 200, 96), (200, 130, 96), (100, 300, 4096), (2560, 2048, 64), (10000, 200, 64), (200, 131, 96), (2560, 2049, 64)]


def operand(r, rows, k, low, high, g):
    pitch = -(-(-(-k // 2)) // 16) * 16
    codes = r.integers(0, 16, (rows, k)).astype(np.uint8)
    codes[rows // 2] = 0                                                  # a row of zeros stays zero whatever the scales are
    scales = r.integers(low, high, (rows, k // 16)).astype(np.uint8)
    sb = np.zeros(Q.scale_bytes(rows, k, 16), np.uint8)
    sb[Q.scale_places(rows, k // 16)] = scales
    dev = lambda a: torch.from_numpy(a).cuda()                            # noqa: E731
    return B.fp4_operand(dev(Q.pack(codes, pitch)), dev(sb), rows, k, 16, torch.full((1,), g, device="cuda")), Q.dequantize(codes, scales, 16, 1.0)


# scale bytes: 0x01 .. 2^-9, 0x18 .. 2^-4, 0x60 .. 2^5, 0x7E = 448
@pytest.mark.parametrize("ga,gb,low,high", [(1e-21, 1e-21, 0x68, 0x78), (3e-5, 1e-37, 0x68, 0x78), (2e19, 2e19, 0x01, 0x04), (3e36, 100.0, 0x01, 0x04),
                                            (0.01, 3e38, 0x01, 0x04), (1e37, 1e-36, 0x18, 0x30), (0.5, 3.0, 0x18, 0x30)])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_of_scales_outside_of_fp32(ga, gb, low, high, m, n, k):
    r = np.random.default_rng(m + n)
    if high == 4 and k > 96:
        k = 96
    oa, a = operand(r, m, k, low, high, ga)
    ob, b = operand(r, n, k, low, high, gb)
    scale = float(np.float32(ga)) * float(np.float32(gb))
    ref, mag = a @ b.T * scale, np.abs(a) @ np.abs(b).T * scale
    assert np.abs(ref).max() < 2.0 ** 127 and np.abs(ref).max() > 2.0 ** -120
    for out in (torch.float32, torch.bfloat16):
        y = torch.full((1, 1, 1, m, n), float("nan"), dtype=out, device="cuda")
        B.lamp_gemm_fp4(oa, ob, y)
        assert B.lamp_get_async_status() == 0
        tol = (76 + k // 64) * 2.0 ** -23 * mag + 2.0 ** -149
        if out is torch.bfloat16:
            tol = tol + 2.0 ** -8 * (np.abs(ref) + tol) + 2.0 ** -134
        got = y.view(m, n).double().cpu().numpy()
        bad = ~(np.abs(got - ref) <= tol)
        assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])
        assert (got[m // 2] == 0).all() and (got[:, n // 2] == 0).all()


@pytest.mark.parametrize("ga,gb", [(float("nan"), 1.0), (1e-25, float("nan")), (float("nan"), 1e30)])
@pytest.mark.parametrize("m,n,k", SHAPES[:4])
def test_a_scale_that_is_nan_stays(ga, gb, m, n, k):
    r = np.random.default_rng(m)
    oa, ob = operand(r, m, k, 0x18, 0x30, ga)[0], operand(r, n, k, 0x18, 0x30, gb)[0]
    y = torch.zeros(1, 1, 1, m, n, device="cuda")
    B.lamp_gemm_fp4(oa, ob, y)
    assert y.isnan().all()
