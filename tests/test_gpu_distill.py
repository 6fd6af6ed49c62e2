"""Top-k distillation loss on the GPU against the fp64 oracle.

Tolerances.  The logits relative to the row's maximum, log p and log q are each formed by at most 4 fp32 operations on numbers
of at most M = max(|z|, |t|) / T + |lse|, so they are off by 8 units of 2^-24 M; the sum of exponentials by 32 units more
(2^-22 per exponential, additions in a tree of <= 64 levels).  ERR = (64 + 8 M) 2^-24 bounds the error of a log and
the relative error of a probability.  A stored bf16 gradient adds 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import pointwise as P
from paper_2006_12575_b200 import binding as B

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, rows, c, k, dt, temp=1.0, tail=False, pitch=None, off=0, weights=True):
        r = np.random.default_rng(seed)
        self.rows, self.c, self.k, self.dt, self.temp = rows, c, k, dt, temp
        z = 2.5 * r.standard_normal((rows, c))
        self.idx = r.integers(0, c, (rows, k)).astype(np.int32)         # duplicates where k is not far below c
        self.t = (3 * r.standard_normal((rows, k))).astype(np.float32)
        for i in range(rows):
            z[i, self.idx[i]] += 0.8 * self.t[i]
        self.w = (r.random(rows) + 0.1).astype(np.float32) if weights else None
        self.buf = torch.full((1, 1, 1, rows, (pitch or c)), 1e4, dtype=dt, device="cuda")
        self.off = off
        self.buf[..., off:off + c] = torch.from_numpy(z).cuda().view(1, 1, 1, rows, c).to(dt)
        self.tlse = None
        if tail:
            self.tlse = (np.log(np.exp(self.t.astype(np.float64) / temp).sum(1)) + 0.3).astype(np.float32)

    def z64(self):
        return self.buf[0, 0, 0, :, self.off:self.off + self.c].double().cpu().numpy()

    def desc(self, buf=None):
        return B.tensor(self.buf if buf is None else buf, self.c, self.off)

    def teacher(self):
        d = lambda a: None if a is None else torch.from_numpy(a).cuda()                  # noqa: E731
        return B.teacher_topk(d(self.idx), d(self.t), self.temp, d(self.tlse))

    def weight(self):
        return None if self.w is None else torch.from_numpy(self.w).cuda()

    def run(self):
        """All three entry points -> (loss_rows, lse, loss, gradient of the fused call, gradient of the two calls)."""
        nan = lambda n: torch.full((n,), float("nan"), device="cuda")                    # noqa: E731
        ws = torch.full((B.lamp_distill_topk_workspace_bytes(self.desc()),), 0xFF, dtype=torch.uint8, device="cuda")
        w, t = self.weight(), self.teacher()
        l1, lse, s1 = nan(self.rows), nan(self.rows), nan(1)
        B.lamp_distill_topk_fwd(self.desc(), t, w, l1, lse, s1, ws)
        g1, g2 = torch.full_like(self.buf, 77.0), torch.full_like(self.buf, 77.0)
        B.lamp_distill_topk_bwd(self.desc(), t, w, lse, self.desc(g1))
        l2, s2 = nan(self.rows), nan(1)
        B.lamp_distill_topk_fwd_bwd(self.desc(), t, w, l2, s2, self.desc(g2), ws)
        assert torch.equal(l1, l2) or torch.isnan(l1).any()
        assert torch.equal(s1, s2) or torch.isnan(s1).any()
        inside = slice(self.off, self.off + self.c)
        for g in (g1, g2):                                             # what lies beside the slice is untouched
            assert (g[..., :self.off] == 77).all() and (g[..., self.off + self.c:] == 77).all()
        return tuple(v.double().cpu().numpy() for v in (l1, lse, s1, g2[0, 0, 0, :, inside], g1[0, 0, 0, :, inside]))

    def check(self, skip=()):
        loss, lse, total, fused, two = self.run()
        z = self.z64()
        w = np.full(self.rows, 1.0 / self.rows) if self.w is None else self.w.astype(np.float64)
        tl = None if self.tlse is None else self.tlse.astype(np.float64)
        rl, rlse, rg = P.distill(z, self.idx, self.t.astype(np.float64), self.temp, w, tl)
        on = np.isfinite(z)
        zm = np.where(on, np.abs(z), 0).max(1)
        tm = np.where(np.isfinite(self.t), np.abs(self.t), 0).max(1)
        err = (64 + 8 * ((zm + tm) / self.temp + np.abs(rlse))) * 2.0 ** -24
        keep = np.array([i for i in range(self.rows) if i not in skip])
        logs = (zm + tm) / self.temp + np.abs(rlse) + 1
        assert (np.abs(lse - rlse) <= err)[keep].all()
        # loss: probabilities (relative err) times log ratios (at most `logs`), and the logs' own error; k terms
        ltol = self.temp ** 2 * (2 * err * (logs + 1) * (1 if tl is None else 1.0))
        assert (np.abs(loss - rl) <= ltol)[keep].all(), np.abs(loss - rl)[keep].max()
        if not skip:
            assert abs(total[0] - (w * rl).sum()) <= (np.abs(w) * ltol).sum() + 2.0 ** -23 * np.abs(w * rl).sum()
        with np.errstate(invalid="ignore", over="ignore"):
            q = np.exp(z / self.temp - rlse[:, None])
        pm = np.zeros_like(q)                                          # probability of the listed classes, for the magnitude
        for i in range(self.rows):
            ok = (self.idx[i] >= 0) & (self.idx[i] < self.c)
            tt = np.where(ok, self.t[i].astype(np.float64) / self.temp, -np.inf)
            if (tt > -np.inf).any():
                p = np.exp(tt - (tl[i] if tl is not None else np.log(np.exp(tt - tt.max()).sum()) + tt.max()))
                np.add.at(pm[i], self.idx[i][ok], p[ok])
        for g, f in ((fused, 1), (two, 2)):
            tol = f * 2 * err[:, None] * np.abs(w)[:, None] * self.temp * (q + pm) + 1e-37
            if self.dt is torch.bfloat16:
                tol = tol + 2.0 ** -8 * (np.abs(rg) + tol)
            bad = ~(np.abs(g - rg) <= tol)[keep]
            assert not bad.any(), (np.argwhere(bad)[:5], g[keep][bad][:5], rg[keep][bad][:5])


SHAPES = [(1, 1, 1), (5, 2, 1), (300, 4, 3), (1000, 10, 4), (77, 16, 16), (33, 31, 5), (40, 33, 40), (3, 100, 7), (70, 257, 64), (9, 1000, 20), (4, 1017, 9),
          (4, 1024, 8), (5, 1025, 8), (3, 4099, 100), (2, 9000, 33), (1, 40000, 10), (2, 130001, 64), (160, 2050, 3), (700, 1500, 5), (400, 6001, 10), (321, 40007, 70), (100, 70000, 5), (77, 32, 32), (600, 20, 33), (700, 128, 32),
          (300, 65, 8), (50, 4344, 100), (30, 2172, 33), (33, 4345, 128), (9, 2173, 129), (3000, 140, 4), (900, 600, 40)]


@pytest.mark.parametrize("rows,c,k", SHAPES)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_loss_and_gradient_match_oracle(rows, c, k, dt):
    Case(rows + c, rows, c, k, dt, temp=[1.0, 2.0, 0.7][rows % 3], tail=rows % 2 == 0, weights=rows % 4 != 1).check()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,pitch,off", [(10, 16, 0), (10, 13, 3), (7, 24, 8), (77, 79, 1), (301, 320, 5), (1001, 1003, 1), (2051, 2063, 2), (20000, 20011, 7)])
def test_slices_of_any_alignment(c, pitch, off, dt):
    Case(c, 6, c, min(c, 9), dt, temp=1.3, pitch=pitch, off=off).check()


@pytest.mark.parametrize("c", [12, 70, 200, 2100, 5000, 70001])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_rows_without_weight_or_entries(c, dt):
    k = Case(c, 9, c, 6, dt, temp=1.5)
    k.w[2] = 0.0
    k.buf[0, 0, 0, 2] = float("nan")                                   # not read: zeros come out
    k.idx[3] = [-1, c, -5, c + 7, 2 ** 31 - 1, -2 ** 31]               # none listed
    k.t[4] = -np.inf
    k.t[5, :5] = -np.inf                                               # one entry left: p = 1
    k.idx[6] = k.idx[6, 0]                                             # the same class six times
    k.idx[7, 1], k.idx[7, 4] = -1, c
    loss, lse, _, fused, two = k.run()
    for r in (2, 3, 4):
        assert loss[r] == 0 and (fused[r] == 0).all() and (two[r] == 0).all()
    assert lse[2] == 0
    k.buf[0, 0, 0, 2] = 0.0
    k.check()


@pytest.mark.parametrize("c", [9, 90, 600, 3000, 50000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_masked_classes_and_rows_that_are_not_finite(c, dt):
    """Logits of -inf and of the type's lowest value (masks), listed and unlisted; +inf and NaN stay in their rows."""
    k = Case(c, 7, c, 4, dt)
    low = torch.finfo(dt).min
    k.idx[:] = np.arange(4)
    b = k.buf[0, 0, 0]
    b[0, 5:8] = float("-inf")
    b[1, 5:8] = low
    b[2, 5:c // 2 + 4] = low
    b[3, 1] = float("-inf")                                            # a listed class the student rules out: loss +inf
    b[4, 6] = float("inf")
    b[5, 7] = float("nan")
    b[6] = float("-inf")
    loss, _, total, fused, two = k.run()
    assert loss[3] == np.inf and np.isfinite(fused[3]).all() and (fused[3, 1] < 0) and np.isfinite(two[3]).all()
    for r in (4, 5, 6):
        assert not np.isfinite(loss[r])
    assert np.isnan(fused[6]).any() and np.isnan(fused[5]).any()
    for r in (0, 1, 2, 3):
        assert np.isfinite(fused[r]).all()
    assert (fused[0, 5:8] == 0).all() and (fused[1, 5:8] == 0).all()
    b[3:] = 0.5
    k.check()


@pytest.mark.parametrize("c", [9, 90, 600, 3000, 50000, 140000])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_row_of_nothing_but_the_lowest_value_is_uniform(c, dt):
    k = Case(c, 3, c, 4, dt)
    k.idx[:] = np.arange(4)
    k.buf[0, 0, 0, 1] = torch.finfo(dt).min
    loss, _, _, fused, _ = k.run()
    t = k.t[1].astype(np.float64)
    logp = t - np.log(np.exp(t).sum())
    ref = (np.exp(logp) * (logp + np.log(c))).sum()
    assert abs(loss[1] - ref) <= 128 * 2.0 ** -24 * (np.abs(t).max() + np.log(c) + 1) * 4
    g = np.full(c, 1.0 / c)
    g[:4] -= np.exp(logp)
    assert (np.abs(fused[1] - k.w[1] * g) <= k.w[1] * (2.0 ** -8 * np.abs(g) + 128 * 2.0 ** -24 * (1.0 / c + (np.arange(c) < 4)))).all()


@pytest.mark.parametrize("rows,c,k", [(1, 400000, 3), (2, 390001, 1024)])
def test_widest_rows(rows, c, k):
    Case(1, rows, c, k, torch.bfloat16, temp=2.0).check()
    Case(2, rows, c // 2, k, torch.float32).check()
    with pytest.raises(B.LampError):
        Case(1, 1, 400001, 1, torch.bfloat16).run()


@pytest.mark.parametrize("rows,c", [(50, 10), (50, 500), (3, 9001), (40, 3001)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gradient_in_place_of_the_logits(rows, c, dt):
    k = Case(rows, rows, c, 8, dt, temp=2.0)
    ws = torch.empty(B.lamp_distill_topk_workspace_bytes(k.desc()), dtype=torch.uint8, device="cuda")
    a, b, loss = torch.empty_like(k.buf), k.buf.clone(), torch.empty(1, device="cuda")
    B.lamp_distill_topk_fwd_bwd(k.desc(), k.teacher(), k.weight(), None, loss, a, ws)
    B.lamp_distill_topk_fwd_bwd(b, k.teacher(), k.weight(), None, None, b)
    assert torch.equal(a, b)
    lse = torch.empty(rows, device="cuda")
    B.lamp_distill_topk_fwd(k.desc(), k.teacher(), None, None, lse)
    b = k.buf.clone()
    B.lamp_distill_topk_bwd(k.desc(), k.teacher(), k.weight(), lse, a)
    B.lamp_distill_topk_bwd(b, k.teacher(), k.weight(), lse, b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("rows,c", [(4000, 10), (300, 700), (2, 60001), (200, 5000)])
def test_repeats_bit_for_bit_on_streams_and_in_graphs(rows, c):
    k = Case(rows, rows, c, 5, torch.bfloat16)
    t, w = k.teacher(), k.weight()
    n = B.lamp_distill_topk_workspace_bytes(k.desc())

    def buffers():
        return torch.full((rows,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda"), torch.empty_like(k.buf), \
            torch.empty(n, dtype=torch.uint8, device="cuda")
    sets = [buffers() for _ in range(4)]
    run = lambda b: B.lamp_distill_topk_fwd_bwd(k.desc(), t, w, b[0], b[1], b[2], b[3])      # noqa: E731
    run(sets[0])
    torch.cuda.synchronize()
    for b in sets[1:3]:
        with torch.cuda.stream(torch.cuda.Stream()):
            run(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(sets[3])
    for _ in range(2):
        sets[3][1].fill_(float("nan"))
        g.replay()
    torch.cuda.synchronize()
    for b in sets[1:]:
        assert all(torch.equal(x, y) for x, y in zip(b[:3], sets[0][:3]))


def test_largest_list_of_entries():
    Case(3, 3, 700, 1024, torch.float32).check()
    Case(5, 9, 700, 512, torch.float32).check()
    Case(4, 2, 5000, 1000, torch.bfloat16, temp=3.0).check()
