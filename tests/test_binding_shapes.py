"""What the binding refuses before any call: matrices of the right size in the wrong order, descriptors of memory on another device (no GPU
needed: the checks look at shapes and device numbers, -1 standing for host memory)."""
import gc
import weakref

import pytest
import torch

from paper_2006_12575_b200 import binding as B


def test_teacher_matrices_have_one_order():
    idx, t = torch.zeros(6, 4, dtype=torch.int32), torch.zeros(6, 4)
    assert B.teacher_topk(idx, t).k == 4 and B.teacher_topk(idx, t, 2.0, torch.zeros(6)).k == 4
    for logits, lse in ((torch.zeros(4, 6), None), (torch.zeros(24), None), (torch.zeros(6, 5), None), (t, torch.zeros(4)), (t, torch.zeros(7))):
        with pytest.raises(ValueError):
            B.teacher_topk(idx, logits, 1.0, lse)


def like(n, c):
    return B.Tensor(4096, B.LAMP_F32, n, 1, 1, 3, c, c, 0)


def test_gate_is_per_sample_then_channel():
    for shape in ((2, 24), (2, 1, 1, 1, 24), (1, 2, 24)):
        B._norm_params(B.block_norm(gate=torch.zeros(shape)), like(2, 24), -1)
    for shape in ((24,), (1, 24), (1, 1, 24)):
        B._norm_params(B.block_norm(gate=torch.zeros(shape)), like(1, 24), -1)
    for shape in ((24, 2), (48,), (3, 16), (2, 12), (4, 12), (24, 1)):
        with pytest.raises(ValueError):
            B._norm_params(B.block_norm(gate=torch.zeros(shape)), like(2, 24), -1)
    with pytest.raises(ValueError):
        B._norm_params(B.block_norm(gate=torch.zeros(2, 24)), like(2, 24), 0)            # host memory, device 0


def test_descriptors_keep_their_memory_and_their_device():
    t = torch.zeros(1, 1, 1, 3, 24)
    d = B.tensor(t, 8, 8)
    alive = weakref.ref(t)
    del t
    gc.collect()
    assert alive() is not None
    assert B._view(d, -1, "x") is d
    with pytest.raises(ValueError):
        B._view(d, 0, "x")
    with pytest.raises(ValueError):
        B._norm_params(B.block_norm(gate_logits=d), like(1, 8), 0)
    bare = like(1, 8)                                                     # built field by field: nothing to check
    assert B._view(bare, 0, "x") is bare
