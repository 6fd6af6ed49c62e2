"""4-bit codes (e2m1) with a scale per block of 32 (e8m0) or 16 (e4m3 times a tensor's scale): what a quantiser has to
write, bit for bit, and the values that an operand stands for in fp64."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
_BORDERS = (VALUES[1:] + VALUES[:-1]) / 2


def e4m3_values():
    """The 128 non-negative e4m3 values by code; 0x7F is NaN."""
    v = np.empty(128)
    for code in range(128):
        e, m = code >> 3, code & 7
        v[code] = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
    v[127] = np.nan
    return v


E4M3 = e4m3_values()


def encode_e4m3(x):
    """Nearest e4m3 code of x >= 0, ties to even, at most 448."""
    x = np.minimum(np.asarray(x, dtype=np.float64), 448.0)
    i = np.searchsorted(E4M3[:127], x)                       # first value >= x
    i = np.clip(i, 1, 126)
    low, high = E4M3[i - 1], E4M3[i]
    up = (x - low > high - x) | ((x - low == high - x) & (i % 2 == 0))
    return np.where(up, i, i - 1).astype(np.uint8)


def encode_e2m1(x):
    """Nearest code 0 .. 15 of x, ties to even, at most 6."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    code = np.zeros(a.shape, dtype=np.uint8)
    for i, b in enumerate(_BORDERS):
        code += (a >= b) if i % 2 else (a > b)               # a tie between codes i and i + 1 goes to the even one
    return code | (np.signbit(x).astype(np.uint8) << 3)


def quantize(x, block, g=1.0):
    """x fp32 [r, k] -> (codes [r, k], scale bytes [r, blocks]).  Every fp32 operation of the definition is one here."""
    x = np.asarray(x, dtype=np.float32)
    r, k = x.shape
    kb = -(-k // block)
    codes, scales = np.zeros((r, k), np.uint8), np.zeros((r, kb), np.uint8)
    for j in range(kb):
        part = x[:, j * block:(j + 1) * block]
        bad = ~np.isfinite(part).all(axis=1)
        with np.errstate(invalid="ignore", over="ignore"):
            amax = np.where(bad, 0, np.abs(part).max(axis=1)).astype(np.float32)
            if block == 32:
                m, e = np.frexp(amax.astype(np.float64))          # amax = m 2^e, m in [1/2, 1): the power of two is 2^(e - 3) up to m = 3/4
                e = np.where(amax > 0, np.where(m <= 0.75, e - 3, e - 2), -127)
                byte = np.clip(e + 127, 0, 254)
                wide = np.ldexp(1.0, byte - 127)
            else:
                byte = encode_e4m3(np.maximum(amax / np.float32(np.float32(6.0) * np.float32(g)), np.float32(2.0 ** -9)))
                wide = (E4M3[byte].astype(np.float32) * np.float32(g)).astype(np.float32)
            v = (part.astype(np.float64) / wide[:, None]) if block == 32 else part / wide[:, None].astype(np.float32)
        codes[:, j * block:(j + 1) * block] = np.where(bad[:, None], 0, encode_e2m1(np.where(bad[:, None], 0, v)))
        scales[:, j] = np.where(bad, 255 if block == 32 else 127, byte)
    return codes, scales


def scale_values(scales, block, g=1.0):
    """fp64 values of scale bytes (NaN codes are NaN); block 16: times g, the product in fp32."""
    if block == 32:
        return np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (E4M3[scales].astype(np.float32) * np.float32(g)).astype(np.float64)


def dequantize(codes, scales, block, g=1.0):
    v = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(scale_values(scales, block, g), block, axis=1)[:, :codes.shape[1]]


def pack(codes, pitch):
    """[r, k] codes -> [r, pitch] bytes, the even position in the low half; what is behind k is 0."""
    r, k = codes.shape
    wide = np.zeros((r, 2 * pitch), np.uint8)
    wide[:, :k] = codes
    return wide[:, 0::2] | (wide[:, 1::2] << 4)


def unpack(q, k):
    return np.stack([q & 15, q >> 4], axis=2).reshape(q.shape[0], -1)[:, :k]


def scale_places(rows, blocks):
    """Index of the scale of (row, block) in an operand's scale bytes: tiles of 128 rows x 4 blocks, [row % 32][row / 32][block % 4] in a tile."""
    out = np.empty((rows, blocks), np.int64)
    tiles = -(-blocks // 4)
    for r in range(rows):
        for i in range(blocks):
            out[r, i] = ((r // 128) * tiles + i // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + i % 4
    return out


def scale_bytes(rows, k, block):
    return -(-rows // 128) * -(-(-(-k // block)) // 4) * 512
