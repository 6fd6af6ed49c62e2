"""Group norm with exactly the scratch that the query asks for: nothing behind it is touched, and the results are those of a larger one."""
import pytest
import torch

from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu
# n, voxels, c, groups: groups and channels that span chunks of channels, one chunk, a cluster's form
SHAPES = [(1, 300, 4096, 1), (2, 3000, 4104, 3), (1, 2000, 6160, 770), (3, 20000, 48, 1), (2, 20000, 48, 48), (1, 200000, 16, 2), (2, 512, 512, 32), (300, 40, 24, 3)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_exact_scratch(shape, dt):
    n, v, c, groups = shape
    g = torch.Generator(device="cuda").manual_seed(v)
    x, dz = (torch.randn(n, 1, 1, v, c, device="cuda", generator=g).to(dt) for _ in range(2))
    p = B.group_norm(groups, None, None, "silu")
    size = B.lamp_group_norm_workspace_bytes(p, x)
    res = []
    for room in (0, 1 << 20):
        ws = torch.full((size + room + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        z, dx = torch.empty_like(x), torch.empty_like(x)
        mr, dw, db = torch.empty(n, groups, 2, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        B.lamp_group_norm_act_fwd(p, x, z, mr, ws[:size + room])
        B.lamp_group_norm_act_bwd(p, dz, x, mr, dx, dw, db, ws[:size + room])
        assert (ws[size:] == 0xA5).all()
        res.append((z, mr, dx, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*res))
    xs = x.view(n, v, groups, -1).double()
    mean = xs.mean((1, 3))
    rstd = 1 / torch.sqrt((xs - mean[:, None, :, None]).square().mean((1, 3)) + 1e-5)
    # sums of at most 256 values in fp32 per thread: 300 roundings of 2^-24 of the deviation, as in the operator's other tests
    assert (res[0][1][..., 0] - mean).abs().max() <= 2.0 ** -24 * 600 * 1.1 and (res[0][1][..., 1] / rstd - 1).abs().max() <= 304 * 2.0 ** -24
