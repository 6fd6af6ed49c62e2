"""fp64 statements of the per-voxel operators: 8-bit blocks, the block norm, the top-k distillation loss.

Plain numpy on matrices [rows, channels]; shares nothing with the CUDA library.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
AMAX_MIN = np.float32(2.0 ** -100)


# --- e4m3 -------------------------------------------------------------------------------------------------------------
def e4m3_table() -> np.ndarray:
    """Value of each of the 256 codes (bias 7, no infinities, 0x7f and 0xff are NaN)."""
    v = np.empty(256)
    for code in range(256):
        s, e, m = code >> 7, (code >> 3) & 15, code & 7
        x = m / 8.0 * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            x = np.nan
        v[code] = -x if s else x
    return v


_TABLE = e4m3_table()
_POSITIVE = _TABLE[:127]                                   # 0 .. 448, ascending


def e4m3_decode(codes: np.ndarray) -> np.ndarray:
    return _TABLE[np.asarray(codes, dtype=np.uint8)]


def e4m3_encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; |x| <= 448 (1 + 2^-20); NaN -> 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a, side="left"), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = np.where(np.signbit(x), code | 0x80, code)
    return np.where(np.isnan(x), 0x7F, code).astype(np.uint8)


def quantize(x: np.ndarray, tile: bool):
    """x [r, k] fp32 values -> (codes [r, k], scales [ceil(k/128), r or ceil(r/128)] fp32), in the fp32 steps of the definition."""
    x = np.asarray(x, dtype=np.float32)
    r, k = x.shape
    kb, rb = -(-k // BLOCK), -(-r // BLOCK)
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), np.float32(0))
    scale = np.empty((kb, rb if tile else r), dtype=np.float32)
    codes = np.empty((r, k), dtype=np.uint8)
    for b in range(kb):
        sl = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
        amax = a[:, sl].max(axis=1)
        if tile:
            amax = np.array([amax[i * BLOCK:(i + 1) * BLOCK].max() for i in range(rb)], dtype=np.float32)
        amax = np.maximum(amax, AMAX_MIN)
        scale[b] = amax * np.float32(1.0 / 448.0)
        inv = np.float32(448.0) / amax
        if tile:
            inv = np.repeat(inv, BLOCK)[:r]
        with np.errstate(invalid="ignore", over="ignore"):
            y = (x[:, sl] * inv[:, None]).astype(np.float64)
        codes[:, sl] = e4m3_encode(np.where(fine[:, sl], y, np.nan))
    return codes, scale


def dequantize(codes: np.ndarray, scale: np.ndarray, tile: bool) -> np.ndarray:
    r, k = codes.shape
    s = np.asarray(scale, dtype=np.float64)
    if tile:
        s = np.repeat(s, BLOCK, axis=1)
    return e4m3_decode(codes) * np.repeat(s[:, :r].T, BLOCK, axis=1)[:, :k]


# --- block norm -------------------------------------------------------------------------------------------------------
def norm(v, w, b, rms, eps):
    """-> (normalised * w + b, normalised, 1 / deviation)."""
    d = v if rms else v - v.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1, keepdims=True) + eps)
    hat = d * rstd
    return hat * w + b, hat, rstd


def norm_backward(dout_w, hat, rstd, rms):
    """Gradient of the normalised row's input; dout_w = gradient times weight."""
    m1 = 0.0 if rms else dout_w.mean(axis=1, keepdims=True)
    return rstd * (dout_w - m1 - hat * (dout_w * hat).mean(axis=1, keepdims=True))


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def block_norm_sum(y, x, post_w, post_b, res, gate, rms, eps):
    """t = x + res * gate * N(y), before it is stored; gate: [rows, c] or 1."""
    return x + res * gate * norm(y, post_w, post_b, rms, eps)[0]


def block_norm_backward(y, t, dout, dh, post_w, post_b, pre_w, res, gate, rms, eps):
    """-> dict of dx, dy, and per row the terms whose sums over rows are the parameters' gradients."""
    out = {}
    dt = np.zeros_like(t) if dout is None else dout.copy()
    if dh is not None:
        _, hat, rstd = norm(t, 1.0, 0.0, rms, eps)
        dt = dt + norm_backward(dh * pre_w, hat, rstd, rms)
        out["pre_w"], out["pre_b"] = dh * hat, dh
    out["dx"] = dt
    if y is not None:
        u, hat, rstd = norm(y, post_w, post_b, rms, eps)
        du = dt * res * gate
        out["dy"] = norm_backward(du * post_w, hat, rstd, rms)
        out["post_w"], out["post_b"], out["res_scale"], out["gate"] = du * hat, du, dt * gate * u, dt * res * u
    return out


# --- distillation -----------------------------------------------------------------------------------------------------
def distill(z, idx, t, temp, weight, tlse=None):
    """-> (loss per row, log-sum per row, gradient of sum_r weight_r loss_r), rows of weight 0 and rows without an entry: 0."""
    rows, c = z.shape
    loss, lse, dz = np.zeros(rows), np.zeros(rows), np.zeros((rows, c))
    for r in range(rows):
        if weight[r] == 0:
            continue
        on = (idx[r] >= 0) & (idx[r] < c)
        ids, tt = idx[r][on], t[r][on] / temp
        if tlse is not None:
            logp = tt - tlse[r]
        else:
            if not on.any() or tt.max() == -np.inf:
                continue
            logp = tt - (tt.max() + np.log(np.exp(tt - tt.max()).sum()))
        p = np.exp(logp)
        if not (p != 0).any():
            continue
        s = z[r] / temp
        top = s.max()
        lse[r] = top + np.log(np.exp(s - top).sum())
        live = p != 0
        loss[r] = temp ** 2 * (p[live] * (logp[live] - (s[ids[live]] - lse[r]))).sum()
        g = np.exp(s - lse[r]) * p.sum()
        np.add.at(g, ids, -p)
        dz[r] = weight[r] * temp * g
    return loss, lse, dz
