"""The gradient written over the logits, where the listed classes of one thread lie in what other threads overwrite: the same bits as
into a buffer of its own, for every form and for long lists."""
import numpy as np
import pytest
import torch

from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,c,k", [(700, 12, 30), (300, 100, 32), (500, 500, 129), (500, 611, 512), (500, 1000, 140), (300, 1000, 1024), (500, 1000, 100),
                                      (400, 600, 33), (60, 1200, 128), (40, 1300, 129), (40, 3001, 500), (3, 60001, 200)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off,beside", [(0, 0), (1, 2)])
def test_backward_in_place_with_long_lists(rows, c, k, dt, off, beside):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + c + k)
    z = torch.randn(1, 1, 1, rows, off + c + beside, device="cuda", generator=g).to(dt)
    idx = torch.randint(0, c, (rows, k), device="cuda", generator=g, dtype=torch.int32)
    teacher = B.teacher_topk(idx, 2 * torch.randn(rows, k, device="cuda", generator=g), 1.5)
    w = torch.rand(rows, device="cuda", generator=g) + 0.1
    view = lambda t: B.tensor(t, c, off)                                                                 # noqa: E731
    lse = torch.empty(rows, device="cuda")
    B.lamp_distill_topk_fwd(view(z), teacher, w, None, lse)
    for call in (lambda a, b: B.lamp_distill_topk_bwd(view(a), teacher, w, lse, view(b)),
                 lambda a, b: B.lamp_distill_topk_fwd_bwd(view(a), teacher, w, None, None, view(b))):
        apart = z.clone()
        call(z, apart)
        for _ in range(20):
            over = z.clone()
            call(over, over)
            assert torch.equal(over, apart)
    assert B.lamp_get_async_status() == 0


@pytest.mark.parametrize("rows,c,k", [(300, 10, 4), (300, 100, 20), (200, 500, 129), (200, 600, 30), (30, 3001, 40), (3, 60001, 20)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gradient_of_another_alignment_than_the_logits(rows, c, k, dt):
    g = torch.Generator(device="cuda")
    g.manual_seed(c)
    z = torch.randn(1, 1, 1, rows, c, device="cuda", generator=g).to(dt)
    idx = torch.randint(0, c, (rows, k), device="cuda", generator=g, dtype=torch.int32)
    teacher = B.teacher_topk(idx, torch.randn(rows, k, device="cuda", generator=g))
    want, loss = torch.empty_like(z), torch.empty(rows, device="cuda")
    B.lamp_distill_topk_fwd_bwd(z, teacher, None, loss, None, want)
    for off, beside in ((1, 0), (3, 2)):
        wide = torch.full((1, 1, 1, rows, off + c + beside), 7.0, dtype=dt, device="cuda")
        B.lamp_distill_topk_fwd_bwd(z, teacher, None, loss, None, B.tensor(wide, c, off))
        got, ref = wide[..., off:off + c].double(), want.double()
        # rows that are not stored as they were read may take another order of work: equal to the last place of the type
        eps = torch.finfo(dt).eps
        assert ((got - ref).abs() <= eps * ref.abs() + 2.0 ** -22 / rows * 3).all()
        assert (wide[..., :off] == 7).all() and (wide[..., off + c:] == 7).all()
