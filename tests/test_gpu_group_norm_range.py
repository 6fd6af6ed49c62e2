"""Group norm of values whose squares are no fp32 numbers: spreads of 1e-30 to 1e35 (eps = 0), and rows masked with the type's lowest value.

The tolerances are those of the operator's other tests: relative to the group's spread, rstd and gradients, whatever their size."""
import numpy as np
import pytest
import torch

from oracle import group as G
from paper_2006_12575_b200 import binding as B
from test_gpu_group_norm import case, check_backward, check_forward, dev, host, scratch

pytestmark = pytest.mark.gpu
# in a cluster's registers, the same with few voxels, streamed
SHAPES = [(2, (5, 6, 7), 48, 6), (2, (1, 1, 3), 16, 16), (1, (26, 26, 26), 24, 3)]
SPREADS = [(0.0, 1e35), (1e31, 1e30), (0.0, 1e20), (-3e9, 1e9), (0.0, 1e-8), (2e-24, 1e-25), (0.0, 1e-30)]
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32), "f32_bf16": (torch.float32, torch.bfloat16)}


def both_ways(shape, x, w, b, dz, types, name, eps):
    n, dhw, c, groups = shape
    xt, zt = TYPES[types]
    tx, tg = dev(x, xt), dev(dz, zt)
    p = B.group_norm(groups, dev(w), dev(b), name, 0.1, eps)
    ws = scratch(p, tx)
    z, mr = torch.empty(x.shape, dtype=zt, device="cuda"), torch.empty(n, groups, 2, device="cuda")
    B.lamp_group_norm_act_fwd(p, tx, z, mr, ws)
    check_forward(z, mr, host(tx), w, b, shape, name, 0.1, eps, zt)
    mean, rstd = G.statistics(host(tx).reshape(n, -1, c), groups, eps)
    mr = dev(np.stack([mean, rstd], 2))
    dx, dw, db = torch.empty_like(tx), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.lamp_group_norm_act_bwd(p, tg, tx, mr, dx, dw, db, ws)
    check_backward(dx, dw, db, host(tg), host(tx), host(mr), w, b, shape, name, 0.1, eps, xt)
    ax, ag = tx.clone(), tg.clone()                                      # in place
    B.lamp_group_norm_act_bwd(p, tg, ax, mr, ax, None, None, ws)
    assert torch.equal(ax, dx)
    if xt is zt:
        B.lamp_group_norm_act_bwd(p, ag, tx, mr, ag, None, None, ws)
        assert torch.equal(ag, dx)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("loc,spread", SPREADS)
@pytest.mark.parametrize("types", list(TYPES))
def test_spreads_of_any_size(shape, loc, spread, types):
    n, dhw, c, groups = shape
    for name in ("silu", "leaky_relu"):
        r, x, w, b = case(shape, 5, loc, spread)
        both_ways(shape, x, w, b, r.standard_normal(x.shape), types, name, 0.0)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2]], ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_channels_of_unlike_spreads(shape, types):
    """Groups of one channel, neighbours 1e40 apart: each thread has all of them."""
    n, dhw, c, _ = shape
    shape = (n, dhw, c, c)
    r, x, w, b = case(shape, 6)
    both_ways(shape, x * 10.0 ** np.tile([0, 20, -20, 12, -12, 30, 4, -4], c // 8), w, b, r.standard_normal(x.shape), types, "gelu", 0.0)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2]], ids=str)
@pytest.mark.parametrize("types", list(TYPES))
def test_rows_masked_with_the_lowest_value(shape, types):
    r, x, w, b = case(shape, 7)
    x.reshape(-1, shape[2])[::23] = torch.finfo(TYPES[types][0]).min
    both_ways(shape, x, w, b, r.standard_normal(x.shape), types, "silu", 1e-5)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2]], ids=str)
def test_one_value_beyond_the_squares(shape):
    """The values that a thread begins with are ordinary, one of the others is not."""
    n, dhw, c, groups = shape
    r, x, w, b = case(shape, 8)
    x[0, -1, -1, -1, 5] = 1e25
    both_ways(shape, x, w, b, r.standard_normal(x.shape), "f32", "none", 1e-5)


@pytest.mark.parametrize("shape", [SHAPES[0], SHAPES[2]], ids=str)
def test_small_deviations_beside_a_small_eps(shape):
    """The squares (1e-40) are below fp32's normal range, and so is eps."""
    r, x, w, b = case(shape, 9, 0.0, 1e-20)
    both_ways(shape, x, w, b, r.standard_normal(x.shape), "f32", "silu", float(np.float32(1e-41)))
