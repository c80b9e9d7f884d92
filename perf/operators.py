"""The operators of a feature encoder (norm, product with its epilogue, gated block) as cases that can be timed and compared.

A case is a dict of plain values; "op" names the operator, "pass" the direction and the rest its sizes and types:

  norm    root-mean-square norm of rows x d with the residual's addition; "serve": output in the type or in 8 bits with
          scales; "train": forward and backward
  linear  act(A W^T + b) + residual, M x K by N x K; "serve" or "train" (forward, then the gradients of A, W and b)
  gated   act(A Wg^T) * (A Wu^T), M x K by twice F x K; "serve" or "train" (forward, then the gradients of A, Wg and Wu)

Types: "f32", "bf16", and for serving "mx8": e4m3 elements, a power-of-two scale for each 32 of a row.  What comes in 8 bits
is made from the plain definition below, so that both sides are given the same codes.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
BLOCK = 32          # elements that share a scale
E4M3_MAX = 448.0    # largest finite e4m3 value


def listed():
    return [
        # one new sample (one token) through the pre-norm of a layer, for 8-bit weights: latency alone
        {"name": "norm_token_mx8", "op": "norm", "pass": "serve", "rows": 1, "d": 2048, "dtype": "bf16", "out": "mx8"},
        # a class of 5000 samples through the same norm, features of 2048
        {"name": "norm_class_mx8", "op": "norm", "pass": "serve", "rows": 5000, "d": 2048, "dtype": "bf16", "out": "mx8"},
        # a training step of a small encoder in fp32, rows and features that are multiples of nothing
        {"name": "norm_train_f32_ragged", "op": "norm", "pass": "train", "rows": 999, "d": 511, "dtype": "f32", "out": "same"},
        # a training step at the large class's size
        {"name": "norm_train_large", "op": "norm", "pass": "train", "rows": 50000, "d": 2048, "dtype": "bf16", "out": "same"},
        # one new sample through a projection: the weights are all there is to read
        {"name": "linear_token", "op": "linear", "pass": "serve", "M": 1, "N": 2048, "K": 2048, "dtype": "bf16", "act": "gelu"},
        # a class of 5000 samples through an 8-bit projection back to the residual stream
        {"name": "linear_class_mx8", "op": "linear", "pass": "serve", "M": 5000, "N": 2048, "K": 8192, "dtype": "mx8", "act": "none"},
        # a training step of a small encoder's head in fp32, odd sizes
        {"name": "linear_train_f32_ragged", "op": "linear", "pass": "train", "M": 999, "N": 511, "K": 300, "dtype": "f32", "act": "relu"},
        # a training step of a projection: 16384 tokens, square weights
        {"name": "linear_train", "op": "linear", "pass": "train", "M": 16384, "N": 2048, "K": 2048, "dtype": "bf16", "act": "gelu"},
        # eight samples served together through a gated block: the two weights are what has to be read
        {"name": "gated_few", "op": "gated", "pass": "serve", "M": 8, "F": 8192, "K": 2048, "dtype": "bf16", "act": "silu"},
        # a class of 5000 samples through a gated block with 8-bit operands
        {"name": "gated_class_mx8", "op": "gated", "pass": "serve", "M": 5000, "F": 8192, "K": 2048, "dtype": "mx8", "act": "silu"},
        # a training step of a small encoder in fp32, features of 512, an inner width that is a multiple of nothing
        {"name": "gated_train_f32_ragged", "op": "gated", "pass": "train", "M": 2500, "F": 1365, "K": 512, "dtype": "f32", "act": "gelu"},
        # the largest: a training step of a gated block, 16384 tokens
        {"name": "gated_train", "op": "gated", "pass": "train", "M": 16384, "F": 8192, "K": 2048, "dtype": "bf16", "act": "silu"},
    ]


def _plain(n):
    """n itself, but 3071 for 3072, a width that no configuration here has."""
    return n - (n == 3072)


def _log_int(rng, lo, hi):
    return _plain(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _size(rng, lo, hi):
    """A length of the range: half of them as model widths come (multiples of 64), half of them anything."""
    n = _log_int(rng, lo, hi)
    return _plain(max(lo, n // 64 * 64)) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["norm", "linear", "linear", "gated", "gated"])
    which = rng.choice(["serve", "train"])
    if op == "norm":
        c = {"op": op, "pass": which, "rows": _log_int(rng, 1, 50000), "d": _size(rng, 64, 8192), "dtype": rng.choice(["f32", "bf16"]),
             "out": "same" if which == "train" else rng.choice(["same", "mx8"])}
        while work(c)["bytes"] > 1.0e9:
            c["rows"] = _plain(c["rows"] // 2 + 1)
        return c
    wide = "N" if op == "linear" else "F"
    c = {"op": op, "pass": which, "M": _log_int(rng, 1 if which == "serve" else 64, 16384), wide: _size(rng, 64, 8192),
         "K": _size(rng, 64, 4096), "dtype": rng.choice(["f32", "bf16", "bf16", "mx8"] if which == "serve" else ["f32", "bf16"]),
         "act": rng.choice(["none", "relu", "silu", "gelu"] if op == "linear" else ["silu", "gelu"])}
    while work(c)["flops"] > (1.0e12 if c["dtype"] == "f32" else 3.2e12):
        c["M"] = _plain(c["M"] // 2 + 1)
    return c


def work(case):
    """What one pass cannot do without: every input read once, every output written once, the products' multiplies and adds."""
    esz = {"f32": 4, "bf16": 2, "mx8": 1 + 1 / BLOCK}[case["dtype"]]
    osz = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n = case["rows"] * case["d"]
        out = 1 + 1 / BLOCK if case["out"] == "mx8" else osz
        if case["pass"] == "serve":      # x, residual -> y, sum
            return {"bytes": n * (3 * osz + out) + case["d"] * osz, "flops": 6 * n}
        return {"bytes": n * 7 * osz + 2 * case["d"] * osz, "flops": 18 * n}     # x, residual, dy, dsum -> y, sum, dx
    M, K, W = case["M"], case["K"], case["N"] if case["op"] == "linear" else case["F"]
    weights = W * K if case["op"] == "linear" else 2 * W * K
    serve = (M * K + weights) * esz + M * W * osz + (M * W + W) * osz * (case["op"] == "linear")
    if case["pass"] == "serve":
        return {"bytes": serve, "flops": 2 * M * weights}
    grads = (M * W + M * K + weights + W * (case["op"] == "linear")) * osz       # dy -> da, dw, db
    return {"bytes": serve + grads, "flops": 6 * M * weights}


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _quantize(v):
    """8 bits with scales, plain: (codes as float8_e4m3fn, scales as float8_e8m0fnu) of the rows of v (fp32)."""
    rows, d = v.shape
    nb = -(-d // BLOCK)
    b = torch.nn.functional.pad(v, (0, nb * BLOCK - d)).reshape(rows, nb, BLOCK)
    m, k = torch.frexp(b.abs().amax(2))              # amax = m 2^k, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(m > 0.875, k - 8, k - 9).clamp(min=-127)
    e = torch.where(m == 0, torch.full_like(e, -127), e)
    q = torch.ldexp(torch.ldexp(b, (-e // 2)[..., None]), (-e - -e // 2)[..., None])
    q = q.reshape(rows, nb * BLOCK)[:, :d].to(torch.float8_e4m3fn).contiguous()
    return q, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(q, scale, dtype):
    """What codes and scales stand for, in `dtype`."""
    e = scale.view(torch.uint8).to(torch.int32) - 127
    s = torch.ldexp(torch.ones((), dtype=dtype, device=q.device), e).repeat_interleave(BLOCK, dim=1)[:, : q.shape[1]]
    return q.to(dtype) * s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def hidden(rows, d, dtype):
        # hidden states: unit variance, one channel in 64 ten times as large, as residual streams have them
        x = torch.randn(rows, d, generator=gen, device="cuda")
        x[:, ::64] *= 10.0
        return x.to(dtype)

    if case["op"] == "norm":
        dt, rows, d = DTYPES[case["dtype"]], case["rows"], case["d"]
        s = {"case": case, "x": hidden(rows, d, dt), "residual": normal(rows, d, dtype=dt), "weight": (1 + 0.1 * normal(d)).to(dt)}
        if case["pass"] == "train":
            s["dy"], s["dsum"] = normal(rows, d, dtype=dt), normal(rows, d, dtype=dt)
        return s
    M, K, W = case["M"], case["K"], case["N"] if case["op"] == "linear" else case["F"]
    mx8 = case["dtype"] == "mx8"
    dt = torch.bfloat16 if mx8 else DTYPES[case["dtype"]]
    s = {"case": case}

    def operand(name, v):
        if mx8:
            s[name], s[name + "_scale"] = _quantize(v)
        else:
            s[name] = v.to(dt)

    operand("a", normal(M, K))
    for name in ("w",) if case["op"] == "linear" else ("w_gate", "w_up"):
        operand(name, normal(W, K, scale=K ** -0.5))
    if case["op"] == "linear":
        s["bias"], s["residual"] = normal(W, scale=0.1, dtype=dt), normal(M, W, dtype=dt)
    if case["pass"] == "train":
        s["dy"] = normal(M, W, dtype=dt)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2211_00839_amd as rcd

    case = s["case"]
    train = case["pass"] == "train"
    if case["op"] == "norm":
        n = rcd.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], quantize=case["out"] == "mx8", want_sum=True,
                         want_rstd=train)
        if not train:
            return {"y": n.y, "sum": n.sum} if n.scale is None else {"y": n.y, "scale": n.scale, "sum": n.sum}
        dx, dweight = rcd.rms_norm_backward(s["dy"], n.sum, n.rstd, s["weight"], dsum=s["dsum"])
        return {"y": n.y, "sum": n.sum, "dx": dx, "dweight": dweight}
    out_dtype = torch.bfloat16 if case["dtype"] == "mx8" else None
    if case["op"] == "linear":
        if not train:
            return rcd.linear(s["a"], s["w"], s["bias"], act=case["act"], residual=s["residual"], a_scale=s.get("a_scale"),
                              w_scale=s.get("w_scale"), out_dtype=out_dtype)
        y, z = rcd.linear(s["a"], s["w"], s["bias"], act=case["act"], residual=s["residual"], want_preact=True)
        da, dw, db = rcd.linear_backward(s["dy"], s["a"], s["w"], z, act=case["act"])
        return {"y": y, "da": da, "dw": dw, "db": db}
    if not train:
        return rcd.gated_linear(s["a"], s["w_gate"], s["w_up"], act=case["act"], a_scale=s.get("a_scale"),
                                gate_scale=s.get("w_gate_scale"), up_scale=s.get("w_up_scale"), out_dtype=out_dtype)
    h, saved = rcd.gated_linear(s["a"], s["w_gate"], s["w_up"], act=case["act"], want_saved=True)
    da, dwg, dwu = rcd.gated_linear_backward(s["dy"], s["a"], s["w_gate"], s["w_up"], saved, act=case["act"])
    return {"y": h, "da": da, "dw_gate": dwg, "dw_up": dwu}


def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return torch.maximum(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))


def _dact(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        t = 1 / (1 + torch.exp(-z))
        return t * (1 + z * (1 - t))
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _run_plain(s):
    case = s["case"]
    train = case["pass"] == "train"
    f = torch.float32
    if case["op"] == "norm":
        dt = s["x"].dtype
        h = s["x"].to(f) + s["residual"].to(f)
        rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        xh = h * rstd
        w = s["weight"].to(f)
        y = xh * w
        if not train:
            if case["out"] == "mx8":
                q, scale = _quantize(y)
                return {"y": q, "scale": scale, "sum": h.to(dt)}
            return {"y": y.to(dt), "sum": h.to(dt)}
        dy = s["dy"].to(f)
        g = dy * w
        dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True)) + s["dsum"].to(f)
        return {"y": y.to(dt), "sum": h.to(dt), "dx": dx.to(dt), "dweight": (dy * xh).sum(0).to(dt)}
    mx8 = case["dtype"] == "mx8"
    dt = torch.bfloat16 if mx8 else s["a"].dtype

    def operand(name):
        return _values(s[name], s[name + "_scale"], f) if mx8 else s[name].to(f)

    a = operand("a")
    if case["op"] == "linear":
        w = operand("w")
        z = a @ w.t() + s["bias"].to(f)
        y = (_act(z, case["act"]) + s["residual"].to(f)).to(dt)
        if not train:
            return y
        dz = s["dy"].to(f) * _dact(z, case["act"])
        return {"y": y, "da": (dz @ w).to(dt), "dw": (dz.t() @ a).to(dt), "db": dz.sum(0).to(dt)}
    wg, wu = operand("w_gate"), operand("w_up")
    g, u = a @ wg.t(), a @ wu.t()
    h = _act(g, case["act"]) * u
    if not train:
        return h.to(dt)
    dh = s["dy"].to(f)
    dg, du = dh * u * _dact(g, case["act"]), dh * _act(g, case["act"])
    return {"y": h.to(dt), "da": (dg @ wg + du @ wu).to(dt), "dw_gate": (dg.t() @ a).to(dt), "dw_up": (du.t() @ a).to(dt)}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    v = {}
    for name, t in s.items():
        if name == "case" or name.endswith("_scale"):
            continue
        v[name] = t.to(torch.float64)
        if name + "_scale" in s:      # value = code * 2^(byte - 127), block by block
            e = s[name + "_scale"].view(torch.uint8).to(torch.float64) - 127
            cols = torch.arange(t.shape[1], device=t.device) // BLOCK
            v[name] = v[name] * torch.pow(2.0, e)[:, cols]
    train = case["pass"] == "train"

    def act_and_slope(z):
        if case["act"] == "none":
            return z, torch.ones_like(z)
        if case["act"] == "relu":
            return z.clamp(min=0), torch.where(z > 0, 1.0, 0.0).double()
        if case["act"] == "silu":
            t = torch.sigmoid(z)
            return z * t, t + z * t * (1 - t)
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)

    if case["op"] == "norm":
        h = v["x"] + v["residual"]
        size = torch.sqrt(h.square().sum(1) / case["d"] + EPS)[:, None]
        y = h / size * v["weight"]
        if not train:
            if case["out"] == "mx8":
                # a code's value before its rounding to 8 bits: the normed value over its block's power of two
                cols = torch.arange(case["d"], device=y.device) // BLOCK
                amax = torch.zeros(y.shape[0], -(-case["d"] // BLOCK), dtype=torch.float64, device=y.device)
                amax.scatter_reduce_(1, cols.expand_as(y), y.abs(), "amax")
                e = torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(min=-127)
                return {"y": y / torch.pow(2.0, e)[:, cols], "scale": torch.pow(2.0, e), "sum": h}
            return {"y": y, "sum": h}
        g = v["dy"] * v["weight"]
        along = (g * h).sum(1, keepdim=True) / case["d"]
        return {"y": y, "sum": h, "dx": g / size - h * along / size ** 3 + v["dsum"], "dweight": (v["dy"] * h / size).sum(0)}
    if case["op"] == "linear":
        z = torch.addmm(v["bias"], v["a"], v["w"].t())
        value, slope = act_and_slope(z)
        y = value + v["residual"]
        if not train:
            return y
        dz = v["dy"] * slope
        return {"y": y, "da": dz @ v["w"], "dw": dz.t() @ v["a"], "db": dz.sum(0)}
    gate, up = v["a"] @ v["w_gate"].t(), v["a"] @ v["w_up"].t()
    value, slope = act_and_slope(gate)
    if not train:
        return value * up
    dgate, dup = v["dy"] * up * slope, v["dy"] * value
    return {"y": value * up, "da": dgate @ v["w_gate"] + dup @ v["w_up"], "dw_gate": dgate.t() @ v["a"], "dw_up": dup.t() @ v["a"]}
