"""The dense side of a training iteration, as cases to time: what a program does beside the tables
with this package's normalization, gradient norm and optimizer.

Ranges the cases stand for:
  adamw       one step over 1-400 tensors of 1 to 3e8 elements together: fp32, or bf16 / fp16 with
              gradients of that type or fp32, with or without fp32 master copies; moments in 32 or
              in 8 bits; tensors of one flat buffer, at any alignment; with and without a clip
              factor; without decay on the vectors
  grad_norm   norm and clip factor of 1-400 tensors of 1 to 6e8 elements together
  layer norm  forward and backward, 1 to 65536 rows of 1 to 16384 elements, odd widths and strides,
              fp32 / bf16 / fp16 with parameters of that type or fp32
The dense side of the package's own workloads (26 one-hot features of 64 floats) is among them; the
other sizes are generic.

8-bit moments.  A tensor's elements are taken in blocks of 128.  With b the exponent field (fp32) of
the block's largest |m| (b >= 14) or v (b >= 30), a moment's code is the upper bits of the fp32 number
|m| 2^(14-b) (a sign, 4 exponent and 3 mantissa bits) or v 2^(30-b) (5 and 3 bits), rounded up or down
by comparing the 20 bits below with a dither of element and step.  A positive v keeps a code above 0.
"""
import math
import random

import torch

own = False

BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
LN_EPS = 1e-5
BLOCK = 128                 # elements of a block of 8-bit moments, to which tensors are padded
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _adamw(name, shape, tensors, total, dtype, grad, bits, master, clip, step, tables=0, dim=0):
    return {"name": name, "op": "adamw", "shape": shape, "tensors": tensors, "total": total,
            "tables": tables, "dim": dim, "dtype": dtype, "grad": grad, "bits": bits,
            "master": master, "clip": clip, "step": step}


def _norm(name, shape, tensors, total, grad, max_norm):
    return {"name": name, "op": "grad_norm", "shape": shape, "tensors": tensors, "total": total,
            "tables": 0, "dim": 0, "dtype": grad, "grad": grad, "max_norm": max_norm}


def _ln(name, op, rows, dim, dtype, params, pad):
    return {"name": name, "op": op, "rows": rows, "dim": dim, "dtype": dtype, "params": params,
            "pad": pad}


def listed():
    return [
        # the dense side of the headline workload (two perceptrons, scale and shift of 26 features
        # of 64 floats), fp32: a step is mostly latency
        _adamw("adamw_f32_dense_side", "dense_side", 0, 0, "f32", "f32", 32, False, False, 10,
               tables=26, dim=64),
        # 16-bit training of a middle-sized model whose tensors have odd sizes: fp32 master copies
        _adamw("adamw_bf16_master_ragged", "ragged", 150, 20_000_000, "bf16", "bf16", 32, True,
               True, 1000),
        # a large model in fp32
        _adamw("adamw_f32_large", "even", 48, 268_435_456, "f32", "f32", 32, False, True, 5),
        # the same dense side with packed moments
        _adamw("adamw8_f32_dense_side", "dense_side", 0, 0, "f32", "f32", 8, False, False, 0,
               tables=26, dim=64),
        # fp16 parameters of odd sizes, gradients accumulated in fp32 and still loss-scaled
        _adamw("adamw8_f16_ragged", "ragged", 150, 20_000_000, "f16", "f32", 8, True, True, 200),
        # a large model in 16 bits with packed moments: what they are for
        _adamw("adamw8_bf16_large", "even", 48, 268_435_456, "bf16", "bf16", 8, False, True, 5000),
        # gradient norm of a small fp32 model
        _norm("grad_norm_f32_ragged", "ragged", 40, 500_000, "f32", 1.0),
        # and of a large one in bf16
        _norm("grad_norm_bf16_large", "even", 96, 536_870_912, "bf16", 1.0),
        # normalization of the bottom perceptron's output, the smallest stated batch
        _ln("ln_fwd_f32_small", "ln_fwd", 128, 64, "f32", "f32", 0),
        # wide rows in bf16
        _ln("ln_fwd_bf16_wide", "ln_fwd", 16_384, 8192, "bf16", "f32", 0),
        # odd width, rows cut out of a wider matrix
        _ln("ln_bwd_f16_odd", "ln_bwd", 10_007, 1001, "f16", "f16", 6),
        # the backward pass of a large batch
        _ln("ln_bwd_bf16_large", "ln_bwd", 32_768, 4096, "bf16", "bf16", 0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["adamw", "adamw", "adamw8", "adamw8", "grad_norm", "ln_fwd", "ln_bwd"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op in ("ln_fwd", "ln_bwd"):
        dim = spread(1, 16_384)
        rows = spread(1, min(65_536, max(1, 120_000_000 // dim)))
        return {"op": op, "rows": rows, "dim": dim, "dtype": dtype,
                "params": rng.choice(["f32", dtype]), "pad": rng.choice([0, 0, 1, 5, 64])}
    tensors = spread(1, 400)
    total = max(tensors, spread(100, 150_000_000))
    case = {"op": "adamw", "shape": rng.choice(["even", "ragged"]), "tensors": tensors,
            "total": total, "tables": 0, "dim": 0, "dtype": dtype,
            "grad": rng.choice(["f32", dtype])}
    if op == "grad_norm":
        case.update(op=op, dtype=case["grad"], max_norm=rng.choice([0.5, 1.0, 1e4]))
        return case
    bits = 8 if op == "adamw8" else 32
    case.update(bits=bits, master=dtype != "f32" and rng.random() < 0.5, clip=rng.random() < 0.5,
                step=spread(1, 20_000) - 1)
    return case


def sizes(case):
    """Elements of the tensors, and which of them are matrices (decayed)."""
    if case["shape"] == "dense_side":
        T, D = case["tables"], case["dim"]
        cross = D + (T + 1) * T // 2
        mats = [(512, 13), (256, 512), (D, 256), (512, cross), (256, 512), (1, 256)]
        out = [(r * c, True) for r, c in mats] + [(r, False) for r, _ in mats]
        return out + [(T * D, False)] * 2
    n, total = case["tensors"], case["total"]
    if case["shape"] == "even":
        each = total // n
        return [(each, True)] * (n - 1) + [(total - each * (n - 1), True)]
    rng = random.Random(n * 1_000_003 + total)
    w = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(n)]
    got = [max(1, int(total * x / sum(w))) for x in w]
    return [(k, i % 3 > 0) for i, k in enumerate(got)]


def _padded(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def _layout(case, device):
    """Where the tensors' elements lie among the moments: None where they lie in order."""
    s = [n for n, _ in sizes(case)]
    if all(n % BLOCK == 0 for n in s):
        return sum(s), None
    n = torch.tensor(s, device=device)
    pad = torch.tensor([_padded(k) for k in s], device=device)
    shift = (pad.cumsum(0) - pad) - (n.cumsum(0) - n)
    pos = torch.arange(int(n.sum()), device=device) + torch.repeat_interleave(shift, n)
    return sum(_padded(k) for k in s), pos


def _cut(flat, case):
    return list(flat.split([n for n, _ in sizes(case)]))


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, device=dev, generator=gen).mul_(scale).add_(shift)

    if case["op"].startswith("ln"):
        rows, dim = case["rows"], case["dim"]
        dt, wt = TYPES[case["dtype"]], TYPES[case["params"]]
        s = {"case": case, "gamma": normal(dim, scale=0.2, shift=1.0).to(wt),
             "beta": normal(dim, scale=0.2).to(wt),
             "x": normal(rows, dim + case["pad"], shift=0.5).to(dt)[:, :dim]}
        if case["op"] == "ln_bwd":
            s["dy"] = normal(rows, dim + case["pad"], scale=0.5).to(dt)[:, :dim]
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = 1 / ((x - s["mean"][:, None]).square_().mean(1) + LN_EPS).sqrt()
            del x
        if own:
            from paper_2404_04270_amd import binding as B
            out = torch.empty(rows, dim, dtype=dt, device=dev)
            if case["op"] == "ln_fwd":
                s["out"] = (out, torch.empty(rows, device=dev), torch.empty(rows, device=dev))
            else:
                s["out"] = (out, torch.empty_like(s["gamma"]), torch.empty_like(s["gamma"]))
                s["ws"] = torch.empty(B.ss_layernorm_rows_workspace_bytes(rows, dim),
                                      dtype=torch.uint8, device=dev)
        return s

    total = sum(n for n, _ in sizes(case))
    g = normal(total).mul_(normal(total).exp_()).mul_(1e-3)
    factor = 0.37
    if case["grad"] == "f16" or case["dtype"] == "f16":
        g, factor = g.mul_(1024), factor / 1024
    s = {"case": case, "g": g.to(TYPES[case["grad"]])}
    del g
    if case["op"] == "grad_norm":
        if own:
            from paper_2404_04270_amd import binding as B
            s["list"] = B.TensorList(_cut(s["g"], case))
            s["clip"] = torch.zeros(4, device=dev)
            s["ws"] = torch.empty(B.ss_grad_norm_workspace_bytes(s["list"]), dtype=torch.uint8,
                                  device=dev)
        return s
    N, pos = _layout(case, dev)
    p = normal(total, scale=0.02)
    s.update(p=p.to(TYPES[case["dtype"]]), pos=pos, step=case["step"], clip=None)
    if case["clip"]:
        s["clip"] = torch.tensor([1.0, factor, 1.0, 0.0], device=dev)
    if case["master"]:
        s["master"] = _place(p, N, pos)
    del p
    decays = torch.tensor([d for _, d in sizes(case)], device=dev)
    if not bool(decays.all()):
        n = torch.tensor([_padded(k) for k, _ in sizes(case)], device=dev)
        s["decay"] = torch.repeat_interleave(decays, n)
    if case["bits"] == 32:
        s["m"] = _place(normal(total, scale=3e-4), N, pos)
        s["v"] = _place(normal(total, scale=1e-3).square_(), N, pos)
    else:
        def codes(lo, hi):
            return torch.randint(lo, hi, (total,), device=dev, generator=gen, dtype=torch.int32)

        sign = codes(0, 2) * 128
        s["m"] = _place((codes(0x38, 0x78) + sign).to(torch.uint8), N, pos)
        del sign
        s["v"] = _place(codes(0xC0, 0xF8).to(torch.uint8), N, pos)
        b = torch.randint(0, 4, (N // BLOCK, 2), device=dev, generator=gen, dtype=torch.int32)
        s["exps"] = (b + torch.tensor([113, 104], device=dev, dtype=torch.int32)).to(torch.uint8)
    if own:
        from paper_2404_04270_amd.optim import AdamW
        params = _cut(s["p"], case)
        opt = AdamW(params, lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                    state_bits=case["bits"], master=case["master"],
                    no_decay=[not d for _, d in sizes(case)],
                    grad_dtypes=[s["g"].dtype] * len(params))
        opt.set_grads(_cut(s["g"], case))
        opt.set_step(s["step"])
        opt.state.m.copy_(s["m"])
        opt.state.v.copy_(s["v"])
        if case["bits"] == 8:
            opt.state.exps.copy_(s["exps"])
            s["moments"] = (torch.empty(N, dtype=torch.bfloat16, device=dev),
                            torch.empty(N, dtype=torch.bfloat16, device=dev))
        if case["master"]:
            opt.state.master.copy_(s["master"])
        s["opt"] = opt
    return s


def _place(x, N, pos):
    if pos is None:
        return x
    out = torch.zeros(N, dtype=x.dtype, device=x.device)
    out[pos] = x
    return out


def _pow2(e):
    """2^e as float64, for whole numbers e."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _bits(x):
    return x.view(torch.int32)


def _mixed(step):
    """The step's part of the dither: 32 bits that change as if drawn from step to step."""
    h = step * 0x9E3779B9 & 0xFFFFFFFF
    h = (h ^ h >> 15) * 0x6A09E667 & 0xFFFFFFFF
    h = (h ^ h >> 13) * 0x9E3779B9 & 0xFFFFFFFF
    return h ^ h >> 16


def _dither(N, step, turn, device):
    u = torch.arange(N, device=device) * 0x6A09E667 + _mixed(step) + turn
    return ((u & 0xFFFFFFFF) >> 12).to(torch.int32)


def _decode(code, exps, top):
    """Values (fp32) of codes without sign; top: the exponent field that a block's largest has."""
    at = exps.to(torch.int64) - top
    x = (code.to(torch.int32) << 20).view(torch.float32).double().view(-1, BLOCK)
    return (x * _pow2(at)[:, None]).float().view(-1)


def _encode(x, top, step, turn):
    """Codes and blocks' exponents of x >= 0 (fp32)."""
    b = (_bits(x.view(-1, BLOCK).amax(1)) >> 23).clamp(min=top)
    y = (x.double().view(-1, BLOCK) * _pow2(top - b)[:, None]).float().view(-1)
    return (_bits(y) + _dither(x.numel(), step, turn, x.device)) >> 20, b


def run(s):
    case = s["case"]
    return {"adamw": _run_adamw, "grad_norm": _run_norm, "ln_fwd": _run_ln_fwd,
            "ln_bwd": _run_ln_bwd}[case["op"]](s, case)


def _run_adamw(s, case):
    packed = case["bits"] == 8
    if own:
        opt = s["opt"]
        opt.step(clip=s["clip"])
        out = {"p": s["p"], "m": opt.state.m, "v": opt.state.v}
        if packed:
            opt.moments(*s["moments"])
            out["m"], out["v"] = s["moments"]
        if case["master"]:
            out["master"] = opt.state.master
        return out
    N, pos, t = s["m"].numel(), s["pos"], s["step"] + 1
    s["step"] = t
    g = _place(s["g"].float(), N, pos)
    if s["clip"] is not None:
        g = g * s["clip"][1]
    p = s["master"] if case["master"] else _place(s["p"].float(), N, pos)
    if packed:
        m = _decode(s["m"] & 127, s["exps"][:, 0], 14) * (1.0 - 2.0 * (s["m"] >> 7))
        v = _decode(s["v"], s["exps"][:, 1], 30)
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    keep = 1 - LR * DECAY
    if "decay" in s:
        keep = torch.where(s["decay"], keep, 1.0)
    size = LR / (1 - BETA1 ** t)
    p = p * keep - size * (m / (v.sqrt() * (1 / math.sqrt(1 - BETA2 ** t)) + EPS))
    s["p"].copy_(p if pos is None else p[pos])
    out = {"p": s["p"]}
    if case["master"]:
        s["master"] = out["master"] = p
    if packed:
        mc, mb = _encode(m.abs(), 14, t, 0)
        vc, vb = _encode(v, 30, t, 1 << 31)
        vc = torch.maximum(vc, (v > 0).to(vc.dtype))
        s["m"] = (mc | (m < 0).to(mc.dtype) << 7).to(torch.uint8)
        s["v"] = vc.to(torch.uint8)
        s["exps"] = torch.stack([mb, vb], 1).to(torch.uint8)
        out["m"] = (_decode(mc, mb, 14) * torch.where(m < 0, -1.0, 1.0)).to(torch.bfloat16)
        out["v"] = _decode(vc, vb, 30).to(torch.bfloat16)
    else:
        s["m"], s["v"] = out["m"], out["v"] = m, v
    return out


def _run_norm(s, case):
    if own:
        from paper_2404_04270_amd import binding as B
        B.ss_grad_norm(s["list"], case["max_norm"], s["clip"], s["ws"])
        return {"norm": s["clip"][0], "factor": s["clip"][1]}
    norm = s["g"].double().square().sum().sqrt()
    return {"norm": norm.float(), "factor": (case["max_norm"] / (norm + 1e-6)).clamp(max=1).float()}


def _run_ln_fwd(s, case):
    if own:
        from paper_2404_04270_amd import binding as B
        B.ss_layernorm_rows_forward(s["x"], None, s["gamma"], s["beta"], LN_EPS, *s["out"])
        y, mean, rstd = s["out"]
        return {"y": y, "mean": mean, "rstd": rstd}
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = 1 / ((x * x).mean(1) + LN_EPS).sqrt()
    y = x * rstd[:, None] * s["gamma"].float() + s["beta"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _run_ln_bwd(s, case):
    if own:
        from paper_2404_04270_amd import binding as B
        dx, dgamma, dbeta = s["out"]
        B.ss_layernorm_rows_backward(s["dy"], s["x"], None, s["gamma"], s["mean"], s["rstd"], dx,
                                     dgamma, dbeta, s["ws"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * rstd
    dgamma, dbeta = (dy * xh).sum(0), dy.sum(0)
    g = dy * s["gamma"].float()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    wt = s["gamma"].dtype
    return {"dx": dx.to(s["x"].dtype), "dgamma": dgamma.to(wt), "dbeta": dbeta.to(wt)}


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"].startswith("ln"):
        n, e, w = case["rows"] * case["dim"], size[case["dtype"]], size[case["params"]]
        if case["op"] == "ln_fwd":
            return {"bytes": 2 * n * e + 8 * case["rows"] + 2 * case["dim"] * w, "flops": 8 * n}
        return {"bytes": 3 * n * e + 8 * case["rows"] + 3 * case["dim"] * w, "flops": 16 * n}
    n, e, ge = sum(k for k, _ in sizes(case)), size[case["dtype"]], size[case["grad"]]
    if case["op"] == "grad_norm":
        return {"bytes": n * ge + 16, "flops": 2 * n}
    each = ge + (e + 8 if case["master"] else 2 * e)
    # moments read and written; packed ones are also given back as values of 16 bits
    each += 16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4
    return {"bytes": n * each, "flops": 15 * n}


# ---- from the definitions, in 64 bits ------------------------------------------------------
def _grid(x, top, above_zero, step, turn, first):
    """x >= 0 (one tensor's, from its place `first` among the moments on) rounded to the numbers that
    8 bits hold: float64 values.  above_zero: a positive x does not become 0."""
    n = x.numel()
    full = torch.zeros(_padded(n), dtype=torch.float64, device=x.device)
    full[:n] = x
    full = full.view(-1, BLOCK)
    most = full.amax(1, keepdim=True)
    # exponent fields as fp32 has them: frexp's exponent is one above
    b = torch.where(most > 0, torch.frexp(most)[1] + 126, 0).clamp(min=top)
    shift = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), (b - top).double())
    y = full / shift                                       # the largest has the exponent field `top`
    field = (torch.frexp(y)[1] + 126).clamp(min=1)
    ulp = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), (field - 130).double())
    i = torch.arange(first, first + full.numel(), device=x.device, dtype=torch.int64)
    h = 2654435769 * step % 2 ** 32
    h = 1779033703 * (h ^ h // 2 ** 15) % 2 ** 32
    h = 2654435769 * (h ^ h // 2 ** 13) % 2 ** 32
    u = (i * 1779033703 + (h ^ h // 2 ** 16) + turn) % 2 ** 32
    k = torch.floor(y / ulp + (u // 4096).double().view_as(y) / (1 << 20))
    k = torch.where((k < 1) & (y > 0) & above_zero, 1.0, k)
    return (k * ulp * shift).view(-1)


def _worth(code, b, top):
    """What codes stand for, by the definition: float64."""
    code = code.to(torch.float64).view(-1, BLOCK)
    field = torch.div(code, 8, rounding_mode="floor")
    mant = code - 8 * field
    two = torch.tensor(2.0, dtype=torch.float64, device=code.device)
    low = torch.pow(two, field.clamp(min=1) - 127)
    value = torch.where(field > 0, (1 + mant / 8) * low, mant / 8 * low)
    return (value * torch.pow(two, b.double() - top)[:, None]).view(-1)


def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    if case["op"].startswith("ln"):
        x, gamma = s["x"].double(), s["gamma"].double()
        mu = x.sum(1, keepdim=True) / case["dim"]
        c = x - mu
        del x
        sd = torch.sqrt((c * c).sum(1, keepdim=True) / case["dim"] + LN_EPS)
        xh = c / sd
        del c
        if case["op"] == "ln_fwd":
            return {"y": gamma * xh + s["beta"].double(), "mean": mu[:, 0], "rstd": 1 / sd[:, 0]}
        dy = s["dy"].double()
        g = gamma * dy
        dx = (g - g.sum(1, keepdim=True) / case["dim"]
              - xh * ((g * xh).sum(1, keepdim=True) / case["dim"])) / sd
        return {"dx": dx, "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    if case["op"] == "grad_norm":
        norm = torch.sqrt(sum((g.double() ** 2).sum() for g in _cut(s["g"], case)))
        return {"norm": norm, "factor": torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0)}
    t = case["step"] + 1
    new_p, new_m, new_v = torch.empty(s["p"].numel(), dtype=torch.float64, device="cuda"), [], []
    factor = 1.0 if s["clip"] is None else float(s["clip"][1])
    masters, first, at = [], 0, 0
    for n, decayed in sizes(case):
        pad = _padded(n)
        grad = s["g"][at:at + n].double() * factor
        old = (s["master"][first:first + n] if case["master"] else s["p"][at:at + n]).double()
        m, v = s["m"][first:first + pad], s["v"][first:first + pad]
        if case["bits"] == 8:
            b = s["exps"][first // BLOCK:(first + pad) // BLOCK]
            sign = 1 - 2 * (m // 128).double()
            m, v = sign * _worth(m % 128, b[:, 0], 14), _worth(v, b[:, 1], 30)
        m = BETA1 * m[:n].double() + (1 - BETA1) * grad
        v = BETA2 * v[:n].double() + (1 - BETA2) * grad ** 2
        p = old * (1 - LR * DECAY * decayed) - LR * (m / (1 - BETA1 ** t)) / (
            torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        new_p[at:at + n] = p
        tail = torch.zeros(pad - n, dtype=torch.float64, device="cuda")
        if case["master"]:
            masters.append(torch.cat([p, tail]))
        if case["bits"] == 8:
            sign = torch.sign(torch.cat([m, tail]))
            m = _grid(m.abs(), 14, False, t, 0, first) * sign
            v = _grid(v, 30, True, t, 1 << 31, first)
        else:
            m, v = torch.cat([m, tail]), torch.cat([v, tail])
        new_m.append(m)
        new_v.append(v)
        at, first = at + n, first + pad
    out = {"p": new_p, "m": torch.cat(new_m), "v": torch.cat(new_v)}
    if case["master"]:
        out["master"] = torch.cat(masters)
    return out
