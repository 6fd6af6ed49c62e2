"""Temperatures that the distillation calls refuse (decided on the host)."""
import ctypes as C

import pytest

from paper_2006_12575_b200 import binding as B

INVALID, UNSUPPORTED = 1, 2


@pytest.mark.parametrize("temp,want", [(2.0 ** -61, UNSUPPORTED), (1e-39, UNSUPPORTED), (1e-45, UNSUPPORTED), (2.0 ** 61, UNSUPPORTED), (1e20, UNSUPPORTED),
                                       (3.4e38, UNSUPPORTED), (0.0, INVALID), (-1.0, INVALID), (float("inf"), INVALID), (float("nan"), INVALID),
                                       (2.0 ** -60, 0), (1.0, 0), (2.0 ** 60, 0)])
def test_temperature_range(temp, want):
    L, t = B.lib(), B.TeacherTopk(4096, 4096, None, 4, temp)
    z = B.Tensor(4096, B.LAMP_BF16, 1, 1, 1, 0 if want == 0 else 6, 16, 16, 0)           # without rows nothing is launched
    r = C.byref
    assert L.lamp_distill_topk_fwd(r(z), r(t), None, 4096, None, None, None, 0, None) == want
    assert L.lamp_distill_topk_bwd(r(z), r(t), None, 4096, r(z), None) == want
    assert L.lamp_distill_topk_fwd_bwd(r(z), r(t), None, None, None, r(z), None, 0, None) == want
