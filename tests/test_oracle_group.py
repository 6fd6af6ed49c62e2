"""Pins of the oracle's group norm and clipping: library special cases in fp64, finite differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import group as G

ACTS = [("none", 0.0), ("leaky_relu", 0.0), ("leaky_relu", 0.1), ("silu", 0.0), ("gelu", 0.0)]


@pytest.mark.parametrize("name,slope", ACTS)
@pytest.mark.parametrize("groups", [1, 3, 12])
def test_forward_and_backward_match_the_library_in_fp64(name, slope, groups):
    r = np.random.default_rng(groups)
    n, v, c = 2, 7, 12
    x, dz, w, b = r.standard_normal((n, v, c)) * 2 + 1, r.standard_normal((n, v, c)), r.standard_normal(c), r.standard_normal(c)
    z, mean, rstd = G.group_norm_act_fwd(x, groups, w, b, name, slope)
    dx, dw, db = G.group_norm_act_bwd(dz, x, mean, rstd, w, b, name, slope)
    tx, tw, tb = (torch.from_numpy(a.copy()).requires_grad_() for a in (x, w, b))
    t = torch.nn.functional.group_norm(tx.transpose(1, 2), groups, tw, tb, 1e-5).transpose(1, 2)
    f = {"none": lambda a: a, "leaky_relu": lambda a: torch.nn.functional.leaky_relu(a, slope), "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu}[name]
    tz = f(t)
    tz.backward(torch.from_numpy(dz))
    for got, ref in ((z, tz), (dx, tx.grad), (dw, tw.grad), (db, tb.grad)):
        np.testing.assert_allclose(got, ref.detach().numpy(), rtol=1e-9, atol=1e-9)


@pytest.mark.parametrize("name,slope", [("silu", 0.0), ("gelu", 0.0), ("none", 0.0)])
def test_backward_is_the_derivative(name, slope):
    r = np.random.default_rng(5)
    n, v, c, groups = 2, 5, 8, 4
    x, dz, w, b = r.standard_normal((n, v, c)), r.standard_normal((n, v, c)), 1 + r.standard_normal(c), r.standard_normal(c)
    _, mean, rstd = G.group_norm_act_fwd(x, groups, w, b, name, slope)
    dx, dw, db = G.group_norm_act_bwd(dz, x, mean, rstd, w, b, name, slope)
    f = lambda a, ww, bb: float((G.group_norm_act_fwd(a, groups, ww, bb, name, slope)[0] * dz).sum())      # noqa: E731
    for arr, grad, put in ((x, dx, lambda d: f(x + d, w, b)), (w, dw, lambda d: f(x, w + d, b)), (b, db, lambda d: f(x, w, b + d))):
        for _ in range(3):
            d = r.standard_normal(arr.shape)
            h = 1e-5
            assert abs((put(h * d) - put(-h * d)) / (2 * h) - float((grad * d).sum())) < 1e-6


def test_statistics_have_moments_zero_and_one_and_are_per_sample():
    r = np.random.default_rng(2)
    x = r.standard_normal((3, 50, 16)) * 5 + 100
    mean, rstd = G.statistics(x, 4, 0.0)
    xhat = G.normalise(x, mean, rstd).reshape(3, 50, 4, 4)
    np.testing.assert_allclose(xhat.mean(axis=(1, 3)), 0, atol=1e-12)
    np.testing.assert_allclose((xhat ** 2).mean(axis=(1, 3)), 1, atol=1e-12)
    alone = G.statistics(x[1:2], 4, 0.0)
    np.testing.assert_array_equal(alone[0][0], mean[1])


def test_clip():
    norm, f, out = G.clip([np.array([3.0]), np.array([0.0, 4.0])], 2.5)
    assert norm == 5.0 and f == 0.5 and out[0][0] == 1.5 and out[1][1] == 2.0
    assert G.clip([np.array([3.0])], 3.0)[1] == 1.0
    assert G.clip([], 1.0)[:2] == (0.0, 1.0)
