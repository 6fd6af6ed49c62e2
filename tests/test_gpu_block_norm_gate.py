"""Gate per element of the block norm at logits of any size, fp32 branch: sigmoid(x) and sigmoid(x) (1 - sigmoid(x)) keep their digits
relative to their own size, on both sides.

Tolerances, u = 2^-24: e^-|x| 4 u, 1 + e one, the reciprocal 2, so g is within 10 u and g (1 - g) within 16 u of its value; the
products around them 8 u more.  The normalised row is within 128 u (1 + A), A = (max |v| + |mean|) / deviation."""
import numpy as np
import pytest
import torch

from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
VALUES = [-80.0, -20.0, -12.0, -5.0, -0.5, 0.0, 0.5, 5.0, 12.0, 16.0, 20.0, 80.0]


@pytest.mark.parametrize("c", [32, 64, 512, 1040])
def test_gate_and_its_gradient_at_large_logits(c):
    r = np.random.default_rng(c)
    rows = len(VALUES) + 20
    logits = np.empty((rows, c), dtype=np.float32)
    logits[:len(VALUES)] = np.array(VALUES, dtype=np.float32)[:, None]
    logits[len(VALUES):] = 10 * r.standard_normal((20, c))
    y, dout = (r.standard_normal((rows, c)).astype(np.float32) for _ in range(2))
    dev = lambda a: torch.from_numpy(a).cuda().view(1, 1, 1, rows, c)                                    # noqa: E731
    p = B.block_norm(gate_logits=dev(logits))
    x, out = torch.zeros(1, 1, 1, rows, c, device="cuda"), torch.empty(1, 1, 1, rows, c, device="cuda")
    B.lamp_block_norm_fwd(p, dev(y), x, out, None)
    dx, dy, dl = (torch.full_like(x, float("nan")) for _ in range(3))
    B.lamp_block_norm_bwd(p, dev(y), x, dev(dout), None, dx, dy, dgate_logits=dl)
    a, z = y.astype(np.float64), logits.astype(np.float64)
    d = a - a.mean(1, keepdims=True)
    sd = np.sqrt((d * d).mean(1, keepdims=True) + 1e-5)
    u = d / sd
    eu = 128 * U * (1 + (np.abs(a).max(1, keepdims=True) + np.abs(a.mean(1, keepdims=True))) / sd)
    g, h = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))                       # h = 1 - g without cancellation
    host = lambda t: t.view(rows, c).double().cpu().numpy()                # noqa: E731
    assert (np.abs(host(out) - g * u) <= g * (eu + 18 * U * np.abs(u)) + 1e-37).all()
    bad = np.abs(host(dl) - dout * u * g * h) > np.abs(dout) * g * h * (eu + 24 * U * np.abs(u)) + 1e-37
    assert not bad.any(), (z[bad][:5], host(dl)[bad][:5], (dout * u * g * h)[bad][:5])


def test_infinite_logits_close_or_open_the_gate():
    c = 64
    y, x, dout = (torch.randn(1, 1, 1, 3, c, device="cuda") for _ in range(3))
    lg = torch.zeros(1, 1, 1, 3, c, device="cuda")
    lg[..., 0, :], lg[..., 1, :] = float("inf"), float("-inf")
    p = B.block_norm(gate_logits=lg)
    out, plain = torch.empty_like(x), torch.empty_like(x)
    B.lamp_block_norm_fwd(p, y, x, out, None)
    B.lamp_block_norm_fwd(B.block_norm(), y, x, plain, None)
    assert torch.equal(out[..., 0, :], plain[..., 0, :]) and torch.equal(out[..., 1, :], x[..., 1, :])
    dx, dy, dl = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    B.lamp_block_norm_bwd(p, y, x, dout, None, dx, dy, dgate_logits=dl)
    assert (dl[..., :2, :] == 0).all() and (dy[..., 1, :] == 0).all() and torch.isfinite(dy).all()
