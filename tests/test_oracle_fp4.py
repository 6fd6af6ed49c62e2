"""Pins of the oracle's 4-bit codes and scales."""
import numpy as np
import pytest
import torch

from oracle import fp4 as Q


def test_e4m3_matches_the_library_type():
    lib = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(Q.E4M3[:127], lib)
    r = np.random.default_rng(0)
    x = np.concatenate([np.exp(r.uniform(-8, 6.09, 4000)), lib, (lib[1:] + lib[:-1]) / 2]).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(Q.encode_e4m3(x), ref)


def test_codes_are_nearest_with_ties_to_even():
    assert [Q.encode_e2m1(np.array([b]))[0] for b in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)] == [0, 2, 2, 4, 4, 6, 6]
    assert Q.encode_e2m1(np.array([-0.0, -5.1, 100.0])).tolist() == [8, 15, 7]
    x = np.random.default_rng(1).uniform(-6, 6, 5000)
    v = Q.VALUES[Q.encode_e2m1(x) & 7] * np.sign(x)
    every = np.concatenate([Q.VALUES, -Q.VALUES])
    np.testing.assert_allclose(np.abs(v - x), np.abs(every[None] - x[:, None]).min(axis=1))


@pytest.mark.parametrize("block", [16, 32])
def test_scales_are_the_smallest_that_hold_a_block(block):
    r = np.random.default_rng(3)
    x = (r.standard_normal((40, 100)) * np.exp(6 * r.standard_normal((40, 1)))).astype(np.float32)
    x[3] = 0
    g = np.float32(2.0 ** -4)
    codes, scales = Q.quantize(x, block, 1.0 if block == 32 else g)
    wide = np.repeat(Q.scale_values(scales, block, g), block, axis=1)[:, :100]
    if block == 32:
        for j in range(4):
            amax = np.abs(x[:, 32 * j:32 * j + 32]).max(axis=1)
            s = wide[:, 32 * j]
            assert (amax <= 6 * s).all() and ((amax > 3 * s) | (s == 2.0 ** -127)).all()
    v = Q.dequantize(codes, scales, block, g)
    # within half a step of the largest codes; blocks of 16: an e4m3 scale rounded down lets the largest value saturate
    sat = (block == 16) & (np.abs(x) > 6 * wide)
    assert (np.abs(v - x) <= wide * (1 + 1e-6))[~sat].all()
    # normal e4m3 scales that are not clipped at 448 are off by at most half a step, 2^-4
    byte = np.repeat(scales, block, axis=1)[:, :100]
    held = (byte >= 8) & (byte < 126)
    assert (np.abs(v - x) <= np.abs(x) / 16 * (1 + 1e-6))[sat & held].all()


def test_packing_and_scale_tiles():
    codes = np.arange(15, dtype=np.uint8).reshape(3, 5)
    q = Q.pack(codes, 16)
    assert q.shape == (3, 16) and q[0, 0] == 0x10 and q[0, 2] == 0x04 and (q[:, 3:] == 0).all()
    np.testing.assert_array_equal(Q.unpack(q, 5), codes)
    p = Q.scale_places(300, 9)
    assert len(np.unique(p)) == p.size and p.max() < Q.scale_bytes(300, 9 * 32, 32) and p[0, 1] == 1 and p[1, 0] == 16 and p[32, 0] == 4 and p[128, 0] == 3 * 512
