"""Pins of the fp64 oracle of the per-voxel operators: known e4m3 values, finite differences of every gradient."""
import numpy as np
import pytest
import torch

from oracle import pointwise as P


def test_e4m3_table_and_rounding():
    assert P.e4m3_decode([0x00, 0x01, 0x08, 0x38, 0x7E, 0x80, 0xB8]).tolist() == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, 0.0, -1.0]
    assert np.isnan(P.e4m3_decode([0x7F, 0xFF])).all()
    codes = np.array([c for c in range(256) if c not in (0x7F, 0xFF)], dtype=np.uint8)
    assert (P.e4m3_encode(P.e4m3_decode(codes)) == codes).all()
    # halfway cases go to the even code, and torch's own conversion agrees on a fine grid
    x = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.1, 0.1, 20001)]).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (P.e4m3_encode(x) == ref).all()


@pytest.mark.parametrize("tile", [False, True])
def test_quantize_is_within_half_a_step(tile):
    r = np.random.default_rng(1)
    x = (r.standard_normal((150, 300)) * np.exp(2 * r.standard_normal((150, 1)))).astype(np.float32)
    x[3] = 0
    q, s = P.quantize(x, tile)
    back = P.dequantize(q, s, tile)
    full = np.repeat(np.repeat(s, 128, axis=1)[:, :150] if tile else s, 128, axis=0)[:300].T
    # half a step: 2^-4 of a normal value, 2^-10 of the scale's unit below 2^-6; the scale itself is rounded (2^-22)
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * full) * (1 + 1e-5)).all()
    assert (q[3] == 0).all()


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gate", ["none", "sample", "element"])
def test_block_norm_backward_is_the_derivative(rms, gate):
    r = np.random.default_rng(2)
    R, C, eps = 6, 16, 1e-3
    y, x, gout, gh = (r.standard_normal((R, C)) for _ in range(4))
    v = dict(post_w=1 + 0.3 * r.standard_normal(C), post_b=r.standard_normal(C), pre_w=1 + 0.3 * r.standard_normal(C),
             pre_b=r.standard_normal(C), res=r.standard_normal(C))
    g_in = {"none": np.zeros(1), "sample": r.standard_normal(C), "element": r.standard_normal((R, C))}[gate]

    def gate_of(g):
        return {"none": 1.0, "sample": g, "element": P.sigmoid(g)}[gate]

    def f(y, x, v, g):
        t = P.block_norm_sum(y, x, v["post_w"], v["post_b"], v["res"], gate_of(g), rms, eps)
        return (t * gout).sum() + (P.norm(t, v["pre_w"], v["pre_b"], rms, eps)[0] * gh).sum()

    t = P.block_norm_sum(y, x, v["post_w"], v["post_b"], v["res"], gate_of(g_in), rms, eps)
    b = P.block_norm_backward(y, t, gout, gh, v["post_w"], v["post_b"], v["pre_w"], v["res"], gate_of(g_in), rms, eps)
    grads = {"y": b["dy"], "x": b["dx"], "post_w": b["post_w"].sum(0), "post_b": b["post_b"].sum(0), "pre_w": b["pre_w"].sum(0),
             "pre_b": b["pre_b"].sum(0), "res": b["res_scale"].sum(0)}
    if gate == "sample":
        grads["g"] = b["gate"].sum(0)
    if gate == "element":
        grads["g"] = b["gate"] * gate_of(g_in) * (1 - gate_of(g_in))
    h = 1e-6
    for name, grad in grads.items():
        for at in [tuple(r.integers(0, n) for n in grad.shape) for _ in range(8)]:
            d = []
            for sgn in (1, -1):
                a = {"y": y.copy(), "x": x.copy(), "g": np.array(g_in, dtype=float), **{k: w.copy() for k, w in v.items()}}
                a[name][at] += sgn * h
                d.append(f(a["y"], a["x"], a, a["g"]))
            assert abs((d[0] - d[1]) / (2 * h) - grad[at]) <= 1e-6 * (1 + abs(grad[at])), (name, at)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_is_the_derivative(tail):
    r = np.random.default_rng(3)
    R, C, K, T = 5, 12, 4, 1.7
    z = 2 * r.standard_normal((R, C))
    idx = r.integers(0, C, (R, K))
    idx[1, 2] = idx[1, 0]                                  # the same class twice
    idx[2, 1], idx[2, 3] = -1, C                           # absent entries
    idx[3] = -7                                            # a row without any
    t = r.standard_normal((R, K))
    t[4, 0] = -np.inf
    w = np.array([0.5, 1.0, 2.0, 1.0, 0.25])
    tl = np.log(np.exp(np.where(np.isinf(t), -50, t) / T).sum(1)) + 0.2 if tail else None
    loss, lse, dz = P.distill(z, idx, t, T, w, tl)
    assert loss[3] == 0 and (dz[3] == 0).all()
    assert np.isfinite(loss).all() and np.isfinite(dz).all()
    if not tail:                                           # a KL divergence, its gradient sums to zero over the classes
        assert (loss >= -1e-12).all() and np.abs(dz.sum(1)).max() < 1e-12
    h = 1e-6
    for i in range(R):
        for j in range(C):
            d = []
            for sgn in (1, -1):
                zz = z.copy()
                zz[i, j] += sgn * h
                d.append((P.distill(zz, idx, t, T, w, tl)[0] * w).sum())
            assert abs((d[0] - d[1]) / (2 * h) - dz[i, j]) < 1e-7
    # a student that equals a teacher listed in full has no loss
    full = np.tile(np.arange(C), (R, 1))
    loss, _, dz = P.distill(z, full, z, T, np.ones(R))
    assert np.abs(loss).max() < 1e-12 and np.abs(dz).max() < 1e-12
