"""Blocks of 16 of the 4-bit quantiser where x / (scale g) or amax / (6 g) leaves the range of fp32: bit for bit against the oracle.

The definition divides in fp32, where such a quotient is infinite: the scale is then the largest (448) and a code the largest of its sign."""
import numpy as np
import pytest
import torch

from oracle import fp4 as Q
from paper_2006_12575_b200 import binding as B

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:overflow encountered")]
TYPES = [torch.bfloat16, torch.float32]
# a tensor's scale times the largest block scale has to be a normal number
SCALES = [0.7, 0.16, 0.1, 2.0 ** -6, 0.01, 1e-3, 1e-6, 1e-12, 1e-20, 1e-27, 1e-30, 1e-35]


def rounded(x, dt):
    with np.errstate(over="ignore"):
        x = np.asarray(x, dtype=np.float32)
    return torch.from_numpy(x).to(dt).float().numpy()


def extremes(r, dt, g):
    """48 rows and columns: blocks with the type's lowest and largest value, with values around 448 * 6 g and around fp32's largest * 6 g,
    beside ordinary ones."""
    big, small = torch.finfo(dt).max, float(np.float32(6) * np.float32(g))
    x = r.standard_normal((48, 48)) * 10.0 ** r.uniform(-3, 3, (48, 1)) * small
    x[0, 3], x[1, 20], x[2, :] = big, -big, -big
    x[3, 40:] = [big, -big, big / 2, -big / 2, 1.0, -1.0, 1e30, -1e30]
    x[4, 5], x[5, 6], x[6, 7] = -1e30, 3e38, -3e38
    for i, f in enumerate([0.5, 0.999, 1.0, 1.001, 2.0, 1e4]):
        x[8 + i, 17], x[16 + i, 17], x[24 + i, 30] = 448 * small * f, -big * min(1.0, small * f), 2.0 ** 127 * min(1.0, small * f)
    return np.clip(rounded(np.clip(x, -big, big), dt), -big, big)


def compare(x, dt, g, transpose):
    rows, c = x.shape
    r, k = (c, rows) if transpose else (rows, c)
    pitch = -(-(-(-k // 2)) // 16) * 16
    q, s = torch.zeros(r, pitch, dtype=torch.uint8, device="cuda"), torch.zeros(Q.scale_bytes(r, k, 16), dtype=torch.uint8, device="cuda")
    op = B.fp4_operand(q, s, r, k, 16, torch.full((1,), float(g), device="cuda"))
    t = torch.from_numpy(x).cuda().to(dt).view(1, 1, 1, rows, c)
    B.lamp_fp4_quantize(t, op, transpose)
    codes, scales = Q.quantize(x.T if transpose else x, 16, g)
    np.testing.assert_array_equal(s.cpu().numpy()[Q.scale_places(r, scales.shape[1])], scales)
    np.testing.assert_array_equal(q.cpu().numpy(), Q.pack(codes, pitch))
    y = torch.empty_like(t)
    B.lamp_fp4_dequantize(op, y, transpose)
    ref = Q.dequantize(codes, scales, 16, g)
    ref = rounded(ref.T.copy() if transpose else ref, dt)
    np.testing.assert_array_equal(y.view(rows, c).float().cpu().numpy(), ref)
    return scales, ref


@pytest.mark.parametrize("g", SCALES)
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("transpose", [False, True])
def test_largest_and_lowest_values(g, dt, transpose):
    x = extremes(np.random.default_rng(1), dt, np.float32(g))
    scales, ref = compare(x, dt, np.float32(g), transpose)
    assert scales.max() == 126 and ref[1, 20] == -ref[0, 3] and ref[1, 20] < 0           # 448, and the sign stays


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("transpose", [False, True])
def test_values_over_the_whole_range(seed, dt, transpose):
    r = np.random.default_rng(seed)
    x = r.standard_normal((80, 96)) * 10.0 ** r.uniform(-36, 38, (80, 96) if seed % 2 else (80, 1))
    big = torch.finfo(dt).max
    g = np.float32(10.0 ** r.uniform(-34, 2))
    compare(np.clip(rounded(np.clip(x, -big, big), dt), -big, big), dt, g, transpose)
