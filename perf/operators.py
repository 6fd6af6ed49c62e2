"""Work items of the 8-bit matrix product, the block normalisation and the distillation loss.

Each case names one call of one operator over a volume's voxels (rows) and channels (columns).  `run` computes it in
elementary torch operations, or, with `own` set, through the library's entry points; `exact` states the same definition
in 64 bits.  Operators:

  quant   x [R, C] -> e4m3 codes and one fp32 scale per block of 128: amax * (1/448) with amax over the block's finite
          values (at least 2^-100), code = round(x * (448 / amax)), NaN where x is not finite.  A block is 128 channels of
          one voxel, or 128 x 128; transposed, the operand is x^T and a block 128 voxels of one channel.
  gemm    y[m, n] = sum_k (qa[m, k] sa[k/128, m]) (qb[n, k] sb[k/128, n or n/128]) + bias[n].
  norm    t = x + r g N1(y), h = N2(t), N LayerNorm or RMS norm over the channels with weight and bias, r a scale per
          channel, g a gate (one per sample and channel, or the sigmoid of a logit per element); t is stored in the type of
          x and h is the norm of the stored t.  Backward: gradients of x, y, the gate and all parameters.
  distill l_r = T^2 sum_j p_j (log p_j - log q_{r, idx_j}), p the softmax of the teacher's k listed logits over T (or
          exp(t / T - lse) with the teacher's own log-sum), q the student's softmax over all classes at T; loss =
          sum_r w_r l_r and its gradient.
"""
import math

import torch

own = False

FP8 = torch.float8_e4m3fn
BLOCK = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def ceil_div(a, b):
    return -(-a // b)


def listed():
    return [
        # activations entering an 8-bit layer: a 64 x 64 x 32 level of the U-Net, 256 channels
        dict(name="quant_rows_level", op="quant", rows=131072, c=256, dt="bf16", transpose=False, tile=False),
        # the same kind of tensor as a weight gradient's operand: blocks along the voxels, odd voxel count
        dict(name="quant_transposed_ragged", op="quant", rows=15 * 17 * 11, c=520, dt="bf16", transpose=True, tile=False),
        # one token through a square layer: the call is bound by reading the weights
        dict(name="gemm_single_token", op="gemm", m=1, n=4096, k=4096, out="bf16", btile=True, bias=False),
        # the deepest level of the five-level U-Net on a 176 x 240 x 128 volume, odd row count, bias
        dict(name="gemm_bottleneck", op="gemm", m=11 * 15 * 8 + 1, n=1024, k=512, out="bf16", btile=True, bias=True),
        # a wide level in a training pass
        dict(name="gemm_wide", op="gemm", m=16384, n=4096, k=4096, out="bf16", btile=True, bias=False),
        # a weight gradient: few outputs, the reduction runs over the voxels, both operands with a scale per row
        dict(name="gemm_weight_gradient", op="gemm", m=512, n=2048, k=32 * 32 * 32 + 40, out="f32", btile=False, bias=False),
        # a handful of tokens: latency
        dict(name="norm_fwd_tokens", op="norm", back=False, n=2, rows=24, c=512, stream="bf16", branch="bf16", rms=False, gate="sample", q=True),
        # a full level, pre-norm written in 8 bits for the next layer
        dict(name="norm_fwd_level", op="norm", back=False, n=2, rows=65536, c=512, stream="bf16", branch="bf16", rms=True, gate="sample", q=True),
        # backward of a level with an fp32 residual stream and a gate per element
        dict(name="norm_bwd_level", op="norm", back=True, n=2, rows=40 * 33 * 31, c=320, stream="f32", branch="bf16", rms=False, gate="element", q=False),
        # segmentation student: ten classes at every voxel of a 128-cube, the teacher's four best
        dict(name="distill_voxels", op="distill", mode="train", rows=128 * 128 * 128, v=10, k=4, dt="f32", temp=2.0, masked=0.1, tail=False),
        # a large vocabulary, odd width, loss and gradient in one pass
        dict(name="distill_vocabulary", op="distill", mode="train", rows=4096, v=50001, k=64, dt="bf16", temp=1.0, masked=0.05, tail=True),
        # evaluation of a few rows: the long axis has to be split
        dict(name="distill_few_rows", op="distill", mode="fwd", rows=5, v=130000, k=20, dt="bf16", temp=1.5, masked=0.0, tail=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quant", "gemm", "gemm", "norm", "norm", "distill", "distill"])
    if op == "quant":
        c = 8 * _log_int(rng, 1, 512)
        rows = _log_int(rng, 1, max(1, 33554432 // c))
        return dict(op=op, rows=rows, c=c, dt=rng.choice(["bf16", "f32"]), transpose=rng.random() < 0.5, tile=rng.random() < 0.4)
    if op == "gemm":
        k = _log_int(rng, 16, 32768)
        n = _log_int(rng, 8, 8192)
        m = _log_int(rng, 1, max(1, min(32768, 16384 * 4096 * 4096 // (n * k), 134217728 // k, 134217728 // n)))
        return dict(op=op, m=m, n=n, k=k, out=rng.choice(["bf16", "f32"]), btile=rng.random() < 0.6, bias=rng.random() < 0.5)
    if op == "norm":
        c = 8 * _log_int(rng, 1, 512)
        n = rng.randint(1, 4)
        rows = _log_int(rng, 1, max(1, 25000000 // (c * n)))
        stream, branch = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        back = rng.random() < 0.5
        return dict(op=op, back=back, n=n, rows=rows, c=c, stream=stream, branch=branch, rms=rng.random() < 0.5,
                    gate=rng.choice(["none", "sample", "element"]), q=(not back) and rng.random() < 0.5)
    mode = rng.choice(["train", "train", "fwd", "bwd"])
    dt = rng.choice(["bf16", "f32"])
    v = rng.randint(2, 40) if rng.random() < 0.35 else _log_int(rng, 41, 200000)
    k = rng.randint(1, min(v, 100))
    rows = _log_int(rng, 1, max(1, min(2097152, 800000000 // (2 * v * (2 if dt == "bf16" else 4) + 8 * k + 12))))
    return dict(op=op, mode=mode, rows=rows, v=v, k=k, dt=dt, temp=rng.choice([1.0, 1.5, 2.0, 4.0]),
                masked=rng.choice([0.0, 0.2]), tail=rng.random() < 0.4)


# ----------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------
def _codes(g, rows, k, tile):
    """An operand in 8 bits as a program holds it: codes [rows, pitch] and scales [blocks of k, rows or blocks of rows]."""
    pitch, kb = ceil_div(k, 16) * 16, ceil_div(k, BLOCK)
    q = (torch.randn(rows, pitch, device="cuda", generator=g) * 90.0).clamp_(-448.0, 448.0).to(FP8)
    per = ceil_div(rows, BLOCK) if tile else rows
    scale = torch.rand(kb, per, device="cuda", generator=g).mul_(0.02).add_(0.005)
    return q, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)                       # noqa: E731
    s = dict(case=dict(case))
    if case["op"] == "quant":
        rows, c = case["rows"], case["c"]
        x = rn(rows, c) * torch.exp(rn(1, c))                                         # channels of unlike ranges
        x[:: 7] = x[:: 7].clamp_min(0.0)
        s["x"] = x.to(DT[case["dt"]]).view(1, 1, 1, rows, c)
        r, k = (c, rows) if case["transpose"] else (rows, c)
        s["q"] = torch.zeros(r, ceil_div(k, 16) * 16, dtype=torch.uint8, device="cuda").view(FP8)
        s["scale"] = torch.zeros(ceil_div(k, BLOCK), ceil_div(r, BLOCK) if case["tile"] else r, device="cuda")
    elif case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        s["qa"], s["sa"] = _codes(g, m, k, False)
        s["qb"], s["sb"] = _codes(g, n, k, case["btile"])
        s["bias"] = rn(n) if case["bias"] else None
        s["y"] = torch.empty(1, 1, 1, m, n, dtype=DT[case["out"]], device="cuda")
    elif case["op"] == "norm":
        n, rows, c = case["n"], case["rows"], case["c"]
        ts, tb = DT[case["stream"]], DT[case["branch"]]
        shape = (n, 1, 1, rows, c)
        s["y"] = (rn(*shape) * 1.5 + 0.3).to(tb)
        s["post_w"], s["post_b"] = 1.0 + 0.2 * rn(c), 0.1 * rn(c)
        s["pre_w"], s["pre_b"] = 1.0 + 0.2 * rn(c), 0.1 * rn(c)
        s["res_scale"] = 0.5 + 0.1 * rn(c)
        s["gate"] = torch.sigmoid(rn(n, c)) if case["gate"] == "sample" else None
        s["logits"] = rn(*shape).to(tb) if case["gate"] == "element" else None
        if case["back"]:
            s["t"] = (rn(*shape) * 2.0 - 0.2).to(ts)
            s["dout"], s["dh"] = rn(*shape).to(ts), rn(*shape).to(tb)
            s["dx"], s["dy"] = torch.empty(shape, dtype=ts, device="cuda"), torch.empty(shape, dtype=tb, device="cuda")
            s["dlogits"] = torch.empty(shape, dtype=tb, device="cuda") if case["gate"] == "element" else None
            for p in ("post_w", "post_b", "pre_w", "pre_b", "res_scale"):
                s["d" + p] = torch.empty(c, device="cuda")
            s["dgate"] = torch.empty(n, c, device="cuda") if case["gate"] == "sample" else None
            # scratch that a program keeps: at most 8 fp32 rows of c per SM and per sample, and some
            s["ws"] = torch.empty(4 * 8 * c * (148 * 8 + n) + 65536, dtype=torch.uint8, device="cuda")
        else:
            s["x"] = (rn(*shape) * 2.0 - 0.2).to(ts)
            s["out"] = torch.empty(shape, dtype=ts, device="cuda")
            s["h"] = torch.empty(shape, dtype=tb, device="cuda") if not case["q"] else None
            if case["q"]:
                s["hq"] = torch.zeros(n * rows, ceil_div(c, 16) * 16, dtype=torch.uint8, device="cuda").view(FP8)
                s["hs"] = torch.zeros(ceil_div(c, BLOCK), n * rows, device="cuda")
    else:
        rows, v, k = case["rows"], case["v"], case["k"]
        start = torch.randint(0, v, (rows, 1), device="cuda", generator=g)
        idx = (start + torch.arange(k, device="cuda") * max(1, v // k)) % v            # k different classes
        t = 9.0 - 5.0 * torch.arange(k, device="cuda") / k + 0.7 * rn(rows, k)
        z = rn(rows, v) * 1.2
        z.scatter_add_(1, idx, 0.8 * t + 0.7 * rn(rows, k))
        s["z"] = z.to(DT[case["dt"]]).view(1, 1, 1, rows, v)
        del z
        s["idx"], s["t"] = idx.to(torch.int32), t.contiguous()
        # the teacher's own log-sum: its listed classes and a tail of about a tenth
        s["tlse"] = torch.logsumexp(t / case["temp"], 1) + 0.1 * torch.rand(rows, device="cuda", generator=g) if case["tail"] else None
        w = torch.full((rows,), 1.0 / rows, device="cuda")
        s["w"] = w.masked_fill_(torch.rand(rows, device="cuda", generator=g) < case["masked"], 0.0) if case["masked"] else w
        s["loss_rows"], s["loss"] = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
        s["lse"] = torch.logsumexp(s["z"].view(rows, v).float() / case["temp"], 1) if case["mode"] == "bwd" else torch.empty(rows, device="cuda")
        s["dz"] = torch.empty_like(s["z"]) if case["mode"] != "fwd" else None
        s["ws"] = torch.empty(8 * rows + 65536, dtype=torch.uint8, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------------------------------
# the library's entry points
# ----------------------------------------------------------------------------------------------------------------------
def _run_own(s):
    from paper_2006_12575_b200 import binding as B
    case = s["case"]
    if case["op"] == "quant":
        rows, c = case["rows"], case["c"]
        r, k = (c, rows) if case["transpose"] else (rows, c)
        B.lamp_fp8_quantize(s["x"], B.fp8_operand(s["q"], s["scale"], r, k, case["tile"]), case["transpose"])
        return {"q": s["q"][:, :k], "scale": s["scale"]}
    if case["op"] == "gemm":
        B.lamp_gemm_fp8(B.fp8_operand(s["qa"], s["sa"], case["m"], case["k"]),
                        B.fp8_operand(s["qb"], s["sb"], case["n"], case["k"], case["btile"]), s["y"], s["bias"])
        return {"y": s["y"]}
    if case["op"] == "norm":
        p = B.block_norm(rms=case["rms"], eps=1e-5, post_w=s["post_w"], post_b=s["post_b"], pre_w=s["pre_w"], pre_b=s["pre_b"],
                         gate=s["gate"], gate_logits=s["logits"], res_scale=s["res_scale"])
        if case["back"]:
            B.lamp_block_norm_bwd(p, s["y"], s["t"], s["dout"], s["dh"], s["dx"], s["dy"], s["ws"], dgate_logits=s["dlogits"],
                                  dpost_w=s["dpost_w"], dpost_b=s["dpost_b"], dpre_w=s["dpre_w"], dpre_b=s["dpre_b"],
                                  dgate=s["dgate"], dres_scale=s["dres_scale"])
            return {n: s[n] for n in ("dx", "dy", "dlogits", "dpost_w", "dpost_b", "dpre_w", "dpre_b", "dgate", "dres_scale")}
        if case["q"]:
            hq = B.fp8_operand(s["hq"], s["hs"], case["n"] * case["rows"], case["c"])
            B.lamp_block_norm_fwd(p, s["y"], s["x"], s["out"], None, hq)
            return {"out": s["out"], "hq": s["hq"][:, :case["c"]], "hs": s["hs"]}
        B.lamp_block_norm_fwd(p, s["y"], s["x"], s["out"], s["h"])
        return {"out": s["out"], "h": s["h"]}
    teacher = B.teacher_topk(s["idx"], s["t"], case["temp"], s["tlse"])
    if case["mode"] == "fwd":
        B.lamp_distill_topk_fwd(s["z"], teacher, s["w"], s["loss_rows"], s["lse"], s["loss"], s["ws"])
        return {"loss": s["loss"], "rows": s["loss_rows"], "lse": s["lse"]}
    if case["mode"] == "bwd":
        B.lamp_distill_topk_bwd(s["z"], teacher, s["w"], s["lse"], s["dz"])
        return {"dz": s["dz"]}
    B.lamp_distill_topk_fwd_bwd(s["z"], teacher, s["w"], s["loss_rows"], s["loss"], s["dz"], s["ws"])
    return {"loss": s["loss"], "rows": s["loss_rows"], "dz": s["dz"]}


# ----------------------------------------------------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------------------------------------------------
def _quantize(x, tile):
    """x fp32 [r, k] -> (codes [r, k], scales [k / 128, r or r / 128])."""
    r, k = x.shape
    kb, rb = ceil_div(k, BLOCK), ceil_div(r, BLOCK)
    fine = torch.isfinite(x)
    a = torch.zeros(rb * BLOCK if tile else r, kb * BLOCK, device=x.device)
    a[:r, :k] = torch.where(fine, x.abs(), torch.zeros_like(x))
    amax = a.view(rb, BLOCK, kb, BLOCK).amax((1, 3)) if tile else a.view(r, kb, BLOCK).amax(2)
    amax = amax.clamp_min(2.0 ** -100)
    inv = torch.full_like(amax, 448.0) / amax
    if tile:
        inv = inv.repeat_interleave(BLOCK, 0)[:r]
    y = x * inv.repeat_interleave(BLOCK, 1)[:, :k]
    q = torch.where(fine, y, torch.full_like(y, math.nan)).to(FP8)
    return q, (amax * torch.tensor(1.0 / 448.0, device=x.device)).t().contiguous()


def _dequantize(q, scale, k, tile, dt=torch.float32):
    r = q.shape[0]
    sc = scale.t().to(dt)
    if tile:
        sc = sc.repeat_interleave(BLOCK, 0)[:r]
    return q[:, :k].to(dt) * sc.repeat_interleave(BLOCK, 1)[:, :k]


def _norm_stats(v, rms, eps):
    mu = torch.zeros_like(v[..., :1]) if rms else v.mean(-1, keepdim=True)
    d = v - mu
    return d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps), 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "quant":
        x = s["x"].view(case["rows"], case["c"]).float()
        q, scale = _quantize(x.t().contiguous() if case["transpose"] else x, case["tile"])
        return {"q": q, "scale": scale}
    if case["op"] == "gemm":
        y = _dequantize(s["qa"], s["sa"], case["k"], False) @ _dequantize(s["qb"], s["sb"], case["k"], case["btile"]).t()
        if s["bias"] is not None:
            y = y + s["bias"]
        return {"y": y.to(DT[case["out"]]).view(1, 1, 1, case["m"], case["n"])}
    if case["op"] == "norm":
        ts, tb, rms = DT[case["stream"]], DT[case["branch"]], case["rms"]
        xh, rstd = _norm_stats(s["y"].float(), rms, 1e-5)
        u = xh * s["post_w"] + s["post_b"]
        n, c = case["n"], case["c"]
        gate = s["gate"].view(n, 1, 1, 1, c) if s["gate"] is not None else torch.sigmoid(s["logits"].float()) if s["logits"] is not None else torch.ones((), device=u.device)
        if not case["back"]:
            out = (s["x"].float() + s["res_scale"] * gate * u).to(ts)
            h = _norm_stats(out.float(), rms, 1e-5)[0] * s["pre_w"] + s["pre_b"]
            if case["q"]:
                q, scale = _quantize(h.view(-1, c), False)
                return {"out": out, "hq": q, "hs": scale}
            return {"out": out, "h": h.to(tb)}
        th, trstd = _norm_stats(s["t"].float(), rms, 1e-5)
        dh = s["dh"].float()
        a = dh * s["pre_w"]
        dt = s["dout"].float() + trstd * (a - (0.0 if rms else a.mean(-1, keepdim=True)) - th * (a * th).mean(-1, keepdim=True))
        du = dt * s["res_scale"] * gate
        b = du * s["post_w"]
        dy = rstd * (b - (0.0 if rms else b.mean(-1, keepdim=True)) - xh * (b * xh).mean(-1, keepdim=True))
        every = (0, 1, 2, 3)
        r = {"dx": dt.to(ts), "dy": dy.to(tb), "dpost_w": (du * xh).sum(every), "dpost_b": du.sum(every), "dpre_w": (dh * th).sum(every),
             "dpre_b": dh.sum(every), "dres_scale": (dt * gate * u).sum(every), "dlogits": None, "dgate": None}
        if case["gate"] == "sample":
            r["dgate"] = (dt * s["res_scale"] * u).sum((1, 2, 3))
        if case["gate"] == "element":
            r["dlogits"] = (dt * s["res_scale"] * u * gate * (1.0 - gate)).to(tb)
        return r
    rows, v, temp = case["rows"], case["v"], case["temp"]
    z = s["z"].view(rows, v).float() / temp
    idx, on = s["idx"].long(), s["w"] != 0
    tt = s["t"] / temp
    tlse = s["tlse"] if s["tlse"] is not None else tt.amax(1) + torch.log(torch.exp(tt - tt.amax(1, keepdim=True)).sum(1))
    logp = tt - tlse[:, None]
    p = torch.exp(logp)
    if case["mode"] == "bwd":
        lse = s["lse"]
    else:
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        rows_loss = torch.where(on, temp * temp * (p * (logp - (z.gather(1, idx) - lse[:, None]))).sum(1), torch.zeros_like(lse))
        loss = (s["w"].double() * rows_loss.double()).sum().float().view(1)
    if case["mode"] == "fwd":
        return {"loss": loss, "rows": rows_loss, "lse": torch.where(on, lse, torch.zeros_like(lse))}
    grad = torch.exp(z - lse[:, None]) * p.sum(1, keepdim=True)
    grad.scatter_add_(1, idx, -p)
    grad = torch.where(on[:, None], grad * (s["w"] * temp)[:, None], torch.zeros_like(grad)).to(s["z"].dtype).view_as(s["z"])
    return {"dz": grad} if case["mode"] == "bwd" else {"loss": loss, "rows": rows_loss, "dz": grad}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------------------------------------------------
# work and 64-bit values
# ----------------------------------------------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "quant":
        e = case["rows"] * case["c"]
        r, k = (case["c"], case["rows"]) if case["transpose"] else (case["rows"], case["c"])
        return {"bytes": e * (size[case["dt"]] + 1) + 4 * ceil_div(k, BLOCK) * (ceil_div(r, BLOCK) if case["tile"] else r), "flops": 2 * e}
    if case["op"] == "gemm":
        m, n, k, kb = case["m"], case["n"], case["k"], ceil_div(case["k"], BLOCK)
        return {"bytes": (m + n) * k + 4 * kb * (m + (ceil_div(n, BLOCK) if case["btile"] else n)) + m * n * size[case["out"]] + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    if case["op"] == "norm":
        e, ss, sb = case["n"] * case["rows"] * case["c"], size[case["stream"]], size[case["branch"]]
        element, par = case["gate"] == "element", 4 * case["c"] * (5 + (case["n"] if case["gate"] == "sample" else 0))
        if case["back"]:
            return {"bytes": e * (3 * ss + 3 * sb + (2 * sb if element else 0)) + 2 * par, "flops": 40 * e}
        h = e + 4 * case["n"] * case["rows"] * ceil_div(case["c"], BLOCK) if case["q"] else e * sb
        return {"bytes": e * (2 * ss + sb + (sb if element else 0)) + h + par, "flops": 20 * e}
    e, rows = case["rows"] * case["v"], case["rows"]
    b = e * size[case["dt"]] * (1 if case["mode"] == "fwd" else 2) + rows * (case["k"] * 8 + 12)
    return {"bytes": int(b), "flops": 6 * e}


def _values64(codes, scales, k, tile):
    """The 64-bit values that codes and scales stand for, block by block of the reduction axis."""
    out = torch.empty(codes.shape[0], k, dtype=torch.float64, device=codes.device)
    for b in range(ceil_div(k, BLOCK)):
        cols = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
        per_row = scales[b].double()
        if tile:
            per_row = per_row[torch.arange(codes.shape[0], device=codes.device) // BLOCK]
        out[:, cols] = codes[:, cols].double() * per_row[:, None]
    return out


def _unit64(v, rms):
    """(normalised v, 1 / deviation) over the last axis, from second moments about the mean."""
    centre = v if rms else v - v.sum(-1, keepdim=True) / v.shape[-1]
    inv = ((centre.square().sum(-1, keepdim=True) / v.shape[-1]) + 1e-5).rsqrt()
    return centre * inv, inv


def _unit64_back(d, unit, inv, rms):
    """Gradient through _unit64: the incoming one less its parts along the constant vector and along `unit`."""
    c = d.shape[-1]
    along = (d * unit).sum(-1, keepdim=True) / c
    level = 0.0 if rms else d.sum(-1, keepdim=True) / c
    return (d - level - unit * along) * inv


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quant":
        x = s["x"].view(case["rows"], case["c"]).double()
        x = x.t() if case["transpose"] else x
        r, k = x.shape
        tall = BLOCK if case["tile"] else 1
        scale = torch.empty(ceil_div(k, BLOCK), ceil_div(r, tall), dtype=torch.float64, device="cuda")
        code = torch.empty(r, k, dtype=torch.float64, device="cuda")
        for b in range(ceil_div(k, BLOCK)):
            cols = slice(b * BLOCK, min(k, (b + 1) * BLOCK))
            big = x[:, cols].abs().amax(1)
            pad = torch.zeros(ceil_div(r, tall) * tall, dtype=torch.float64, device="cuda")
            pad[:r] = big
            scale[b] = pad.view(-1, tall).amax(1).clamp_min(2.0 ** -100) / 448.0
            code[:, cols] = x[:, cols] / scale[b].repeat_interleave(tall)[:r, None]
        # a code is the scaled value rounded to four significant bits (steps of 2^-9 below 2^-6)
        step = torch.exp2(torch.floor(torch.log2(code.abs().clamp_min(2.0 ** -6))) - 3)
        return {"q": torch.round(code / step) * step, "scale": scale}
    if case["op"] == "gemm":
        y = torch.matmul(_values64(s["qa"], s["sa"], case["k"], False), _values64(s["qb"], s["sb"], case["k"], case["btile"]).T)
        return {"y": (y if s["bias"] is None else y + s["bias"].double()).view(1, 1, 1, case["m"], case["n"])}
    if case["op"] == "norm":
        n, c, rms = case["n"], case["c"], case["rms"]
        wide = {key: val.double() for key, val in s.items() if torch.is_tensor(val) and val.is_floating_point() and val.dtype != FP8}
        unit, inv = _unit64(wide["y"], rms)
        branch = unit * wide["post_w"] + wide["post_b"]
        if case["gate"] == "sample":
            open_ = wide["gate"][:, None, None, None, :].expand_as(branch)
        elif case["gate"] == "element":
            open_ = 1.0 / (1.0 + torch.exp(-wide["logits"]))
        else:
            open_ = torch.ones_like(branch)
        factor = open_ * wide["res_scale"]
        if not case["back"]:
            total = wide["x"] + factor * branch
            stored = total.to(DT[case["stream"]]).double()                  # the norm in front of the next block reads this
            nxt = _unit64(stored, rms)[0] * wide["pre_w"] + wide["pre_b"]
            if not case["q"]:
                return {"out": total, "h": nxt}
            flat = nxt.view(-1, c)
            scale = torch.stack([flat[:, b:b + BLOCK].abs().amax(1) / 448.0 for b in range(0, c, BLOCK)])
            return {"out": total, "hq": flat / scale.repeat_interleave(BLOCK, 0)[:c].t(), "hs": scale}
        tunit, tinv = _unit64(wide["t"], rms)
        d_total = wide["dout"] + _unit64_back(wide["dh"] * wide["pre_w"], tunit, tinv, rms)
        d_branch = d_total * factor
        flat = lambda v: v.reshape(-1, c).sum(0)                                                     # noqa: E731
        res = {"dx": d_total, "dy": _unit64_back(d_branch * wide["post_w"], unit, inv, rms), "dpost_w": flat(d_branch * unit),
               "dpost_b": flat(d_branch), "dpre_w": flat(wide["dh"] * tunit), "dpre_b": flat(wide["dh"]),
               "dres_scale": flat(d_total * open_ * branch), "dgate": None, "dlogits": None}
        through = d_total * wide["res_scale"] * branch
        if case["gate"] == "sample":
            res["dgate"] = through.reshape(n, -1, c).sum(1)
        if case["gate"] == "element":
            res["dlogits"] = through * open_ * (1.0 - open_)
        return res
    rows, v, temp = case["rows"], case["v"], case["temp"]
    idx, weight = s["idx"].long(), s["w"].double()
    teacher = s["t"].double() / temp
    teacher = teacher - (s["tlse"].double()[:, None] if s["tlse"] is not None else torch.logsumexp(teacher, 1, keepdim=True))
    mass = torch.exp(teacher)
    student = s["z"].view(rows, v).double() / temp
    norm = s["lse"].double() if case["mode"] == "bwd" else torch.logsumexp(student, 1)
    student -= norm[:, None]
    kl = (mass * (teacher - torch.gather(student, 1, idx))).sum(1) * temp ** 2
    kl = torch.where(weight == 0, torch.zeros_like(kl), kl)
    loss = torch.dot(kl, weight).view(1)
    if case["mode"] == "fwd":
        return {"loss": loss, "rows": kl, "lse": torch.where(weight == 0, torch.zeros_like(norm), norm)}
    slope = student.exp_().mul_(mass.sum(1, keepdim=True)).scatter_add_(1, idx, -mass).mul_((weight * temp)[:, None])
    slope = slope.view(1, 1, 1, rows, v)
    return {"dz": slope} if case["mode"] == "bwd" else {"loss": loss, "rows": kl, "dz": slope}
