"""Work items of the group norm with an activation, the clipping of gradients by their global norm, and the 4-bit layers.

Each case names one call of one operator.  `run` computes it in elementary torch operations, or, with `own` set, through the
library's entry points; `exact` states the same definition in 64 bits.  Operators:

  gnorm   z = act(t), t = (x - mean_g) / sqrt(var_g + eps) * w[c] + b[c], with mean and biased variance of a sample's group of
          channels over its voxels; act: none, leaky ReLU (slope 0: ReLU), SiLU, GELU (erf).  Backward: gradients of x, w and b.
  clip    norm = sqrt(sum of squares over all tensors), factor = 1 where norm <= max_norm, else max_norm / norm; every tensor
          times factor.
  quant4  x [R, C] -> 4-bit codes (e2m1: 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives) and one 8-bit scale per block along the
          channels (transposed: along the voxels), and back to the values they stand for.  Blocks of 32: scale = the
          smallest power of two with amax <= 6 scale.  Blocks of 16: scale = e4m3(amax / (6 g)), at least 2^-9, times the
          tensor's scale g.  code = nearest, ties to even, of x / scale.
  gemm4   y[m, n] = sum_k a[m, k] b[n, k] + bias[n] of two operands in that form.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
FP8 = torch.float8_e4m3fn
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5


def ceil_div(a, b):
    return -(-a // b)


def listed():
    return [
        # deepest level of a five-level U-Net on two 128-cubes: latency
        dict(name="gnorm_fwd_deep", op="gnorm", back=False, n=2, rows=8 * 8 * 8, c=512, groups=32, act="silu", dt="bf16"),
        # top level of a wide network on a 128-cube
        dict(name="gnorm_fwd_top", op="gnorm", back=False, n=1, rows=128 * 128 * 128, c=64, groups=8, act="silu", dt="bf16"),
        # a ragged level in fp32 whose groups (ten channels) do not match the vectors
        dict(name="gnorm_bwd_ragged", op="gnorm", back=True, n=2, rows=40 * 33 * 31, c=320, groups=32, act="gelu", dt="f32"),
        # top level of the 32-filter network in training
        dict(name="gnorm_bwd_top", op="gnorm", back=True, n=1, rows=128 * 128 * 128, c=32, groups=4, act="relu", dt="bf16"),
        # vectors of a network's norms and biases: many tensors of a few elements
        dict(name="clip_vectors", op="clip", count=62, size=512, spread=1.0, kind="f32", ratio=0.25),
        # gradients of a 32 .. 512 filter network (22 million), layer by layer
        dict(name="clip_network", op="clip", count=46, size=492000, spread=1.5, kind="f32", ratio=0.1),
        # a large network: fp32 and bf16 gradients side by side
        dict(name="clip_large", op="clip", count=301, size=700001, spread=0.5, kind="mixed", ratio=0.5),
        # activations entering a 4-bit layer, and back to the values a check or a straight-through estimator reads
        dict(name="quant4_rows_level", op="quant4", rows=131072, c=256, dt="bf16", block=32, transpose=False),
        # operand of a weight gradient: blocks along the voxels, odd voxel count
        dict(name="quant4_transposed_ragged", op="quant4", rows=15 * 17 * 11, c=520, dt="bf16", block=16, transpose=True),
        # one token through a square layer
        dict(name="gemm4_single_token", op="gemm4", m=1, n=4096, k=4096, out="bf16", block=16, bias=False),
        # the deepest level of the five-level U-Net on a 176 x 240 x 128 volume, odd row count, bias
        dict(name="gemm4_bottleneck", op="gemm4", m=11 * 15 * 8 + 1, n=1024, k=512, out="bf16", block=32, bias=True),
        # a wide level in a training pass
        dict(name="gemm4_wide", op="gemm4", m=16384, n=4096, k=4096, out="bf16", block=16, bias=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gnorm", "gnorm", "gnorm", "clip", "clip", "quant4", "gemm4", "gemm4"])
    if op == "gnorm":
        c = 8 * _log_int(rng, 1, 256)
        n = rng.randint(1, 4)
        back, dt = rng.random() < 0.5, rng.choice(["bf16", "bf16", "f32"])
        rows = _log_int(rng, 1, max(1, (48000000 if back else 100000000) // (c * n * (1 if dt == "bf16" else 2))))
        groups = rng.choice([g for g in range(1, c + 1) if c % g == 0])
        return dict(op=op, back=back, n=n, rows=rows, c=c, groups=groups, act=rng.choice(["none", "relu", "leaky", "silu", "gelu"]), dt=dt)
    if op == "clip":
        count = _log_int(rng, 1, 400)
        return dict(op=op, count=count, size=_log_int(rng, 1, 100000000 // count), spread=rng.choice([0.0, 0.5, 1.0]),
                    kind=rng.choice(["f32", "bf16", "mixed"]), ratio=rng.choice([0.01, 0.5, 2.0]))
    if op == "quant4":
        c = 8 * _log_int(rng, 1, 512)
        return dict(op=op, rows=_log_int(rng, 1, 33554432 // c), c=c, dt=rng.choice(["bf16", "f32"]), block=rng.choice([16, 32]),
                    transpose=rng.random() < 0.5)
    k = _log_int(rng, 16, 32768)
    n = _log_int(rng, 8, 8192)
    m = _log_int(rng, 1, max(1, min(32768, 16384 * 4096 * 4096 // (n * k), 134217728 // k, 134217728 // n)))
    return dict(op=op, m=m, n=n, k=k, out=rng.choice(["bf16", "f32"]), block=rng.choice([16, 32]), bias=rng.random() < 0.5)


# ----------------------------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------------------------
def _scale_at(rows, kb, device="cuda"):
    """Place of the scale of (row, block) in an operand's scale bytes: tiles of 128 rows x 4 blocks."""
    r = torch.arange(rows, device=device)[:, None]
    j = torch.arange(kb, device=device)[None, :]
    return ((r // 128) * ceil_div(kb, 4) + j // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + j % 4


def _scale_bytes(rows, k, block):
    return ceil_div(rows, 128) * ceil_div(ceil_div(k, block), 4) * 512


def _pack(code):
    """Codes [r, k] in 0 .. 15 -> bytes [r, pitch], the even position in the low half."""
    r, k = code.shape
    pitch = ceil_div(ceil_div(k, 2), 16) * 16
    wide = torch.zeros(r, 2 * pitch, dtype=torch.uint8, device=code.device)
    wide[:, :k] = code
    return wide[:, 0::2] | (wide[:, 1::2] << 4)


def _sizes(case):
    """The tensors' sizes, spread about `size` in a fixed manner; the types alternate where `kind` is mixed."""
    count, size, spread = case["count"], case["size"], case["spread"]
    f = [math.exp(spread * math.cos(1.0 + 2.4 * i)) for i in range(count)]
    total = size * count / sum(f)
    return [(max(1, int(total * w)), "bf16" if case["kind"] == "bf16" or (case["kind"] == "mixed" and i % 2) else "f32") for i, w in enumerate(f)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    rn = lambda *s: torch.randn(*s, device="cuda", generator=g)                       # noqa: E731
    s = dict(case=dict(case))
    if case["op"] == "gnorm":
        n, rows, c, groups, dt = case["n"], case["rows"], case["c"], case["groups"], DT[case["dt"]]
        shape = (n, 1, 1, rows, c)
        x = rn(*shape)
        x.mul_(0.5 + torch.rand(c, device="cuda", generator=g)).add_(0.5 * rn(c))      # channels of unlike ranges
        s["x"] = x.to(dt)
        del x
        s["w"], s["b"] = 1.0 + 0.2 * rn(c), 0.1 * rn(c)
        s["mean_rstd"] = torch.empty(n, groups, 2, device="cuda")
        if case["back"]:
            s["dz"], s["dx"] = rn(*shape).to(dt), torch.empty(shape, dtype=dt, device="cuda")
            s["dw"], s["db"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            # what the forward pass left behind
            flat = s["x"].view(n, rows, groups, c // groups)
            mean = flat.double().sum((1, 3)) / (rows * c // groups)
            var = torch.stack([(flat[i].double() - mean[i, None, :, None]).square_().sum((0, 2)) for i in range(n)]) / (rows * c // groups)
            s["mean_rstd"] = torch.stack([mean, 1.0 / torch.sqrt(var + EPS)], 2).float()
        else:
            s["z"] = torch.empty(shape, dtype=dt, device="cuda")
        # scratch that a program keeps: partial sums per channel of a few hundred CTAs
        s["ws"] = torch.empty(16 * c * n * 640 + 65536, dtype=torch.uint8, device="cuda")
    elif case["op"] == "clip":
        sizes = _sizes(case)
        s["flat"], s["out"], s["parts"], s["outs"] = {}, {}, [], []
        for kind in ("f32", "bf16"):
            total = sum(m for m, t in sizes if t == kind)
            if total:
                v = torch.empty(total, dtype=DT[kind], device="cuda")
                step = 1 << 26
                for i in range(0, total, step):
                    v[i:i + step] = rn(min(step, total - i)) * 0.01
                s["flat"][kind], s["out"][kind] = v, torch.empty_like(v)
        at = dict(f32=0, bf16=0)
        for m, kind in sizes:
            s["parts"].append(s["flat"][kind][at[kind]:at[kind] + m])
            s["outs"].append(s["out"][kind][at[kind]:at[kind] + m])
            at[kind] += m
        s["max_norm"] = case["ratio"] * 0.01 * math.sqrt(sum(m for m, _ in sizes))
        s["norm"], s["factor"] = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        s["ws"] = torch.empty(65536 + 64 * len(sizes), dtype=torch.uint8, device="cuda")
        if own:                                                              # the list of tensors that a program keeps
            from paper_2006_12575_b200 import binding as B
            s["list"] = B.grad_list(s["parts"], s["outs"])
    elif case["op"] == "quant4":
        rows, c, block = case["rows"], case["c"], case["block"]
        x = rn(rows, c) * torch.exp(rn(1, c))                                         # channels of unlike ranges
        x[:: 7] = x[:: 7].clamp_min(0.0)
        s["x"] = x.to(DT[case["dt"]]).view(1, 1, 1, rows, c)
        del x
        s["y"] = torch.empty_like(s["x"])
        r, k = (c, rows) if case["transpose"] else (rows, c)
        s["q"] = torch.zeros(r, ceil_div(ceil_div(k, 2), 16) * 16, dtype=torch.uint8, device="cuda")
        s["scale"] = torch.zeros(_scale_bytes(r, k, block), dtype=torch.uint8, device="cuda")
        # the tensor's scale puts the largest block scale at e4m3's largest value; a power of two, as a program that shifts it would keep
        s["g"] = torch.exp2(torch.ceil(torch.log2(s["x"].float().abs().amax() / 2688.0))).view(1) if block == 16 else None
    else:
        m, n, k, block = case["m"], case["n"], case["k"], case["block"]
        for name, rows in (("a", m), ("b", n)):
            x = rn(rows, k)
            gs = torch.full((1,), 0.01, device="cuda") if block == 16 else None
            code, scale = _quantize(x, block, gs)
            del x
            s["q" + name], s["g" + name] = _pack(code), gs
            sb = torch.zeros(_scale_bytes(rows, k, block), dtype=torch.uint8, device="cuda")
            sb[_scale_at(rows, ceil_div(k, block))] = scale
            s["s" + name] = sb
        s["bias"] = rn(n) if case["bias"] else None
        s["y"] = torch.empty(1, 1, 1, m, n, dtype=DT[case["out"]], device="cuda")
    return s


# ----------------------------------------------------------------------------------------------------------------------
# the library's entry points
# ----------------------------------------------------------------------------------------------------------------------
def _run_own(s):
    from paper_2006_12575_b200 import binding as B
    case = s["case"]
    if case["op"] == "gnorm":
        act, slope = {"relu": ("leaky_relu", 0.0), "leaky": ("leaky_relu", 0.01)}.get(case["act"], (case["act"], 0.0))
        p = B.group_norm(case["groups"], s["w"], s["b"], act, slope, EPS)
        if case["back"]:
            B.lamp_group_norm_act_bwd(p, s["dz"], s["x"], s["mean_rstd"], s["dx"], s["dw"], s["db"], s["ws"])
            return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
        B.lamp_group_norm_act_fwd(p, s["x"], s["z"], s["mean_rstd"], s["ws"])
        return {"z": s["z"], "mean_rstd": s["mean_rstd"]}
    if case["op"] == "clip":
        B.lamp_grad_clip(s["list"], s["max_norm"], s["norm"], s["factor"], s["ws"])
        return {"norm": s["norm"], "factor": s["factor"], "out": s["out"]}
    if case["op"] == "quant4":
        r, k = (case["c"], case["rows"]) if case["transpose"] else (case["rows"], case["c"])
        op = B.fp4_operand(s["q"], s["scale"], r, k, case["block"], s["g"])
        B.lamp_fp4_quantize(s["x"], op, case["transpose"])
        B.lamp_fp4_dequantize(op, s["y"], case["transpose"])
        return {"y": s["y"]}
    B.lamp_gemm_fp4(B.fp4_operand(s["qa"], s["sa"], case["m"], case["k"], case["block"], s["ga"]),
                    B.fp4_operand(s["qb"], s["sb"], case["n"], case["k"], case["block"], s["gb"]), s["y"], s["bias"])
    return {"y": s["y"]}


# ----------------------------------------------------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------------------------------------------------
def _quantize(x, block, g):
    """x fp32 [r, k] -> (codes 0 .. 15 [r, k], scale bytes [r, k / block])."""
    r, k = x.shape
    kb = ceil_div(k, block)
    a = torch.zeros(r, kb * block, device=x.device)
    a[:, :k] = x.abs()
    amax = a.view(r, kb, block).amax(2)
    del a
    if block == 32:
        mant, e = torch.frexp(amax)                                          # amax = mant 2^e, mant in [0.5, 1)
        e = torch.where(mant <= 0.75, e - 3, e - 2).clamp(-127, 127)         # 6 * 2^(e - 3) = 0.75 * 2^e
        e = torch.where(amax > 0, e, torch.full_like(e, -127))
        scale, wide = (e + 127).to(torch.uint8), torch.ldexp(torch.ones((), device=x.device), e)
    else:
        s8 = (amax / (6.0 * g)).clamp(2.0 ** -9, 448.0).to(FP8)
        scale, wide = s8.view(torch.uint8), s8.float() * g
    v = x.abs() / wide.repeat_interleave(block, 1)[:, :k]
    code = torch.zeros(r, k, dtype=torch.uint8, device=x.device)
    # borders between neighbouring codes; a tie goes to the even code
    for i, b in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (v >= b) if i % 2 else (v > b)
    return code | (torch.signbit(x).to(torch.uint8) << 3), scale


def _codes(q, k):
    """Bytes [r, pitch] -> the codes [r, k]."""
    c = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1)
    return c[:, :k]


def _dequantize(q, sb, k, block, g):
    r, kb = q.shape[0], ceil_div(k, block)
    return _code_values(_codes(q, k), sb[_scale_at(r, kb)], block, g)


def _code_values(code, scale, block, g):
    k = code.shape[1]
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    wide = torch.exp2(scale.float() - 127.0) if block == 32 else scale.view(FP8).float() * g
    return table[code.int()] * wide.repeat_interleave(block, 1)[:, :k]


def _act(t, act):
    if act in ("relu", "leaky"):
        return torch.where(t > 0, t, t * (0.01 if act == "leaky" else 0.0))
    if act == "silu":
        return t / (1.0 + torch.exp(-t))
    return 0.5 * t * (1.0 + torch.erf(t * math.sqrt(0.5))) if act == "gelu" else t


def _slope(t, act):
    if act in ("relu", "leaky"):
        return torch.where(t > 0, torch.ones_like(t), torch.full_like(t, 0.01 if act == "leaky" else 0.0))
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-t))
        return sig * (1.0 + t * (1.0 - sig))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(t * math.sqrt(0.5))) + t * torch.exp(-0.5 * t * t) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(t)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "gnorm":
        n, rows, c, groups, dt = case["n"], case["rows"], case["c"], case["groups"], DT[case["dt"]]
        x = s["x"].view(n, rows, groups, c // groups).float()
        w, b = s["w"].view(1, 1, groups, -1), s["b"].view(1, 1, groups, -1)
        if not case["back"]:
            mean = x.mean((1, 3), keepdim=True)
            d = x - mean
            rstd = 1.0 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
            z = _act(d * rstd * w + b, case["act"])
            return {"z": z.to(dt).view_as(s["x"]), "mean_rstd": torch.stack([mean.view(n, groups), rstd.view(n, groups)], 2)}
        mean, rstd = s["mean_rstd"][..., 0].view(n, 1, groups, 1), s["mean_rstd"][..., 1].view(n, 1, groups, 1)
        xh = (x - mean) * rstd
        dy = s["dz"].view_as(x).float() * _slope(xh * w + b, case["act"])
        wd = dy * w
        dx = rstd * (wd - wd.mean((1, 3), keepdim=True) - xh * (wd * xh).mean((1, 3), keepdim=True))
        return {"dx": dx.to(dt).view_as(s["x"]), "dw": (dy * xh).sum((0, 1)).view(c), "db": dy.sum((0, 1)).view(c)}
    if case["op"] == "clip":
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for p in s["parts"]:
            total = total + (p.float() * p.float()).sum().double()
        norm = torch.sqrt(total).float().view(1)
        factor = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm)
        for p, o in zip(s["parts"], s["outs"]):
            o.copy_(p.float() * factor)
        return {"norm": norm, "factor": factor, "out": s["out"]}
    if case["op"] == "quant4":
        x = s["x"].view(case["rows"], case["c"]).float()
        if case["transpose"]:
            x = x.t().contiguous()
        code, scale = _quantize(x, case["block"], s["g"])
        del x
        y = _code_values(code, scale, case["block"], s["g"])
        return {"y": (y.t() if case["transpose"] else y).to(DT[case["dt"]]).contiguous().view_as(s["x"])}
    y = _dequantize(s["qa"], s["sa"], case["k"], case["block"], s["ga"]) @ _dequantize(s["qb"], s["sb"], case["k"], case["block"], s["gb"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(DT[case["out"]]).view_as(s["y"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------------------------------------------------
# work and 64-bit values
# ----------------------------------------------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    if case["op"] == "gnorm":
        e, es = case["n"] * case["rows"] * case["c"], size[case["dt"]]
        if case["back"]:
            return {"bytes": 3 * e * es + 16 * case["c"] + 8 * case["n"] * case["groups"], "flops": 20 * e}
        return {"bytes": 2 * e * es + 8 * case["c"] + 8 * case["n"] * case["groups"], "flops": 12 * e}
    if case["op"] == "clip":
        sizes = _sizes(case)
        return {"bytes": sum(2 * m * size[t] for m, t in sizes) + 8, "flops": 3 * sum(m for m, _ in sizes)}
    if case["op"] == "quant4":
        e = case["rows"] * case["c"]
        r, k = (case["c"], case["rows"]) if case["transpose"] else (case["rows"], case["c"])
        held = r * ceil_div(k, 2) + r * ceil_div(k, case["block"])
        return {"bytes": 2 * e * size[case["dt"]] + 2 * held, "flops": 4 * e}
    m, n, k = case["m"], case["n"], case["k"]
    held = (m + n) * (ceil_div(k, 2) + ceil_div(k, case["block"]))
    return {"bytes": held + m * n * size[case["out"]] + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}


def _act64(t, act):
    """(act(t), its derivative)"""
    if act == "none":
        return t, torch.ones_like(t)
    if act == "silu":
        open_ = torch.sigmoid(t)
        return t * open_, open_ + t * open_ * torch.sigmoid(-t)
    if act == "gelu":
        below = 0.5 * torch.erfc(-t / math.sqrt(2.0))
        return t * below, below + t * torch.exp(-t.square() / 2) / math.sqrt(2 * math.pi)
    k = torch.full_like(t, 0.01 if act == "leaky" else 0.0)
    k[t > 0] = 1.0
    return t * k, k


def _held64(q, sb, rows, k, block, g):
    """The 64-bit values of a packed operand, one block of the reduction axis at a time."""
    out = torch.empty(rows, k, dtype=torch.float64, device=q.device)
    row = torch.arange(rows, device=q.device)
    tiles = ceil_div(ceil_div(k, block), 4)
    magnitude = torch.tensor(E2M1, dtype=torch.float64, device=q.device)
    for j in range(ceil_div(k, block)):
        byte = sb[(row.div(128, rounding_mode="floor") * tiles + j // 4) * 512 + row.remainder(32) * 16 + row.remainder(128).div(32, rounding_mode="floor") * 4 + j % 4]
        scale = torch.exp2(byte.double() - 127) if block == 32 else byte.view(FP8).double() * g.double()
        for i in range(j * block, min(k, (j + 1) * block)):
            nibble = (q[:, i // 2].int() >> (4 * (i & 1))) & 15
            out[:, i] = torch.where(nibble >= 8, -scale, scale) * magnitude[(nibble & 7).long()]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "gnorm":
        n, rows, c, groups = case["n"], case["rows"], case["c"], case["groups"]
        per = c // groups
        res = {"z": torch.empty(n, rows, c, dtype=torch.float64, device="cuda"), "mean_rstd": torch.empty(n, groups, 2, dtype=torch.float64, device="cuda")}
        if case["back"]:
            res = {"dx": torch.empty(n, rows, c, dtype=torch.float64, device="cuda"), "dw": torch.zeros(c, dtype=torch.float64, device="cuda"),
                   "db": torch.zeros(c, dtype=torch.float64, device="cuda")}
        xs = s["x"].view(n, rows, c)
        for i in range(n):
            for g0 in range(0, groups, max(1, 64 // per)):                   # a slice of whole groups at a time
                g1 = min(groups, g0 + max(1, 64 // per))
                ch = slice(g0 * per, g1 * per)
                x = xs[i, :, ch].double().view(rows, g1 - g0, per)
                w, b = s["w"][ch].double().view(1, -1, per), s["b"][ch].double().view(1, -1, per)
                if case["back"]:
                    mean, rstd = s["mean_rstd"][i, g0:g1].double().unbind(1)
                else:
                    count = rows * per
                    mean = x.sum((0, 2)) / count
                    rstd = ((x - mean[:, None]).square().sum((0, 2)) / count + EPS).rsqrt()
                unit = (x - mean[:, None]) * rstd[:, None]
                value, slope = _act64(unit * w + b, case["act"])
                if not case["back"]:
                    res["z"][i, :, ch] = value.view(rows, -1)
                    res["mean_rstd"][i, g0:g1] = torch.stack([mean, rstd], 1)
                    continue
                slope *= s["dz"].view(n, rows, c)[i, :, ch].double().view_as(x)
                res["db"][ch] += slope.sum(0).view(-1)
                res["dw"][ch] += (slope * unit).sum(0).view(-1)
                slope *= w
                level, along = slope.sum((0, 2)) / (rows * per), (slope * unit).sum((0, 2)) / (rows * per)
                res["dx"][i, :, ch] = ((slope - level[:, None] - unit * along[:, None]) * rstd[:, None]).view(rows, -1)
        for name in ("z", "dx"):
            if name in res:
                res[name] = res[name].view(n, 1, 1, rows, c)
        return res
    if case["op"] == "clip":
        total = sum(float(torch.dot(p.double(), p.double())) for p in s["parts"])
        norm = math.sqrt(total)
        factor = 1.0 if norm <= s["max_norm"] else s["max_norm"] / norm
        one = lambda v: torch.full((1,), v, dtype=torch.float64, device="cuda")           # noqa: E731
        return {"norm": one(norm), "factor": one(factor), "out": {t: v.double() * factor for t, v in s["flat"].items()}}
    if case["op"] == "quant4":
        rows, c, block = case["rows"], case["c"], case["block"]
        x = s["x"].view(rows, c)
        x = (x.t() if case["transpose"] else x).double()
        r, k = x.shape
        y = torch.empty_like(x)
        for j in range(0, k, block):
            part = x[:, j:j + block]
            big = part.abs().amax(1, keepdim=True)
            if block == 32:
                scale = torch.exp2(torch.ceil(torch.log2(torch.clamp_min(big, 2.0 ** -140) / 6.0)).clamp(-127, 127))
                scale = torch.where(scale * 3.0 >= big, torch.where(scale > 2.0 ** -127, scale / 2, scale), scale)   # the logarithm's rounding
            else:
                g = s["g"].double()
                v = (big / (6.0 * g)).clamp(2.0 ** -9, 448.0)
                step = torch.exp2(torch.floor(torch.log2(v)).clamp_min(-6) - 3)                 # four significant bits
                scale = torch.round(v / step) * step * g
            v = part / scale
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(1.0))).clamp_max(2) - 1)  # two significant bits
            y[:, j:j + block] = (torch.round(v / step) * step).clamp(-6.0, 6.0) * scale
        return {"y": (y.t().contiguous() if case["transpose"] else y).view(1, 1, 1, rows, c)}
    if case["k"] > 40000:
        return None
    a = _held64(s["qa"], s["sa"], case["m"], case["k"], case["block"], s["ga"])
    b = _held64(s["qb"], s["sb"], case["n"], case["k"], case["block"], s["gb"])
    y = torch.matmul(a, b.T)
    return {"y": (y if s["bias"] is None else y + s["bias"].double()).view(1, 1, 1, case["m"], case["n"])}
