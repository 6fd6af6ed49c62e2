"""Scratch of the group norm: what the groups need, not what as many groups as channels would (no GPU needed)."""
import ctypes as C

import pytest

from paper_2006_12575_b200 import binding as B


def need(groups, c, voxels, n=1):
    x = B.Tensor(4096, B.LAMP_BF16, n, 1, 1, voxels, c, c, 0)
    return B.lib().lamp_group_norm_workspace_bytes(C.byref(B.GroupNorm(groups, 0, 0.0, 1e-5, None, None)), C.byref(x))


# a pair of fp64 per channel and part backward, at most 18 parts and their sum here; 600 MB had been asked for
def test_many_channels_in_few_groups():
    assert 0 < need(8, 65536, 4608) <= 16 * 65536 * 20


@pytest.mark.parametrize("c,voxels,n", [(8, 1, 1), (64, 100000, 2), (4096, 5000, 1), (65536, 4608, 1)])
def test_scratch_grows_with_the_groups(c, voxels, n):
    sizes = [need(g, c, voxels, n) for g in (1, c // 8, c)]
    assert sizes == sorted(sizes) and sizes[0] >= 16 * n * c                     # the channels' sums of the backward pass in any case
