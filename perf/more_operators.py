"""Attention of the feature encoder (what mixes a sample's tokens) as cases that can be timed and compared.

  out = softmax(scale Q K^T + bias[bucket(key's position - query's position)]) V

for each head, with its gradients.  A case is a dict of plain values:

  pass      "serve": attention alone; "train": attention, then the gradients of q, k, v and of the bias table
  form      "dense": batch x length; "cache": few new tokens against keys of which each sequence has a length of its own;
            "padded": dense, the keys behind each sequence's length are padding; "ragged": sequences of different
            lengths one after the other, as views of one projection's result
  heads, kv_heads, D, causal; buckets (0: no bias) and distance: the learned bias of relative positions
  mix       with lengths of their own: what they are made from

The queries of a sequence stand at the end of its keys.  Types: "f32", "bf16".
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(which, form, dtype, B, Tq, Tk, heads, kv_heads, D, causal, buckets=0, distance=128, mix=0):
    return {"pass": which, "form": form, "dtype": dtype, "B": B, "Tq": Tq, "Tk": Tk, "heads": heads, "kv_heads": kv_heads, "D": D,
            "causal": causal, "buckets": buckets, "distance": distance, "mix": mix}


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)

    return [
        # one new token of one short sample: latency alone
        named("serve_token", "serve", "dense", "bf16", 1, 1, 300, 8, 8, 64, True),
        # one new token of a very long document, keys and values shared by eight heads: reading them is all there is
        named("serve_token_long", "serve", "dense", "bf16", 1, 1, 100003, 16, 2, 128, True),
        # one new token of each of 64 sequences that are served together, lengths of 1 to 4096, with the bias
        named("serve_tokens_cache", "serve", "cache", "bf16", 64, 1, 4096, 16, 4, 128, True, buckets=32, mix=1),
        # five queries that look at the tokens of another text, fp32, sizes that are multiples of nothing
        named("serve_few_f32", "serve", "dense", "f32", 2, 5, 777, 6, 3, 40, False, buckets=18, distance=50),
        # 256 samples of up to 512 tokens encoded together
        named("serve_samples", "serve", "ragged", "bf16", 256, 512, 512, 8, 8, 64, False, buckets=32, mix=2),
        # a long document read through at once
        named("serve_document", "serve", "dense", "bf16", 1, 16384, 16384, 16, 4, 128, True),
        # a training step of a small encoder in fp32: a few short samples, odd head size
        named("train_f32_ragged", "train", "ragged", "f32", 7, 333, 333, 4, 2, 40, False, buckets=32, mix=3),
        # a training step on a padded batch of a few hundred tokens each
        named("train_padded", "train", "padded", "bf16", 32, 197, 197, 12, 12, 64, False, mix=4),
        # a training step on samples of up to 512 tokens, one after the other
        named("train_samples", "train", "ragged", "bf16", 100, 512, 512, 8, 8, 64, False, buckets=32, mix=5),
        # a training step of an encoder of texts, every head with its bias
        named("train_texts", "train", "dense", "bf16", 4, 2048, 2048, 16, 16, 64, False, buckets=32),
        # a training step of a causal model, keys and values shared by four heads
        named("train_causal", "train", "dense", "bf16", 4, 4096, 4096, 16, 4, 128, True),
        # the largest: a training step on long texts
        named("train_long", "train", "dense", "bf16", 2, 8192, 8192, 16, 16, 128, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    which = rng.choice(["serve", "train"])
    form = rng.choice(["dense", "cache", "ragged"] if which == "serve" else ["dense", "padded", "ragged"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4])
    D = rng.choice([64, 64, 128, 128, 8 * rng.randint(2, 16), rng.randint(16, 128)])
    causal = rng.random() < 0.5
    Tk = _log_int(rng, 1, 8192)
    Tq = _log_int(rng, 1, min(Tk, 16)) if form == "cache" else Tk if form != "dense" or rng.random() < 0.6 else _log_int(rng, 1, 8192)
    buckets = rng.choice([0, 0, 2 * rng.randint(4, 32)])
    c = _case(which, form, dtype, _log_int(rng, 1, 256), Tq, Tk, heads, kv_heads, D, causal, buckets, rng.randint(40, 300), rng.randint(1, 10 ** 6))
    while work(c)["flops"] > (2.0e11 if dtype == "f32" else 3.5e12) or work(c)["bytes"] > 5.0e8:
        if c["B"] > 1:
            c["B"] = (c["B"] + 1) // 2
        else:
            c["Tq"], c["Tk"] = (c["Tq"] + 1) // 2, (c["Tk"] + 1) // 2
    return c


def _lengths(case):
    """[(queries, keys)] of the sequences."""
    B, Tq, Tk = case["B"], case["Tq"], case["Tk"]
    if case["form"] == "dense":
        return [(Tq, Tk)] * B
    rng = random.Random(case["mix"])
    least = Tq if case["form"] == "cache" else 1
    some = [_log_int(rng, least, Tk) for _ in range(B)]
    some[rng.randrange(B)] = Tk
    if case["form"] == "ragged":
        return [(n, n) for n in some]
    return [(Tq, n) for n in some]


def _pairs(tq, tk, causal):
    """How many (query, key) pairs are not masked."""
    if not causal:
        return tq * tk
    seen = min(tq, tk)                       # queries that see a key: they see tk - seen + 1 .. tk of them
    return seen * tk - seen * (seen - 1) // 2


def work(case):
    """What one pass cannot do without: inputs read once, outputs written once; two products forward and five backward."""
    lengths = _lengths(case)
    esz = 4 if case["dtype"] == "f32" else 2
    H, KV, D = case["heads"], case["kv_heads"], case["D"]
    q, k = sum(a for a, _ in lengths) * H * D * esz, sum(b for _, b in lengths) * KV * D * esz
    table = case["buckets"] * H * esz
    pairs = sum(_pairs(a, b, case["causal"]) for a, b in lengths) * H
    if case["pass"] == "serve":
        return {"bytes": 2 * q + 2 * k + table, "flops": 4 * D * pairs}
    return {"bytes": 4 * q + 4 * k + 2 * table, "flops": 14 * D * pairs}     # q, k, v, dout -> out, dq, dk, dv


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, H, KV, D = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["D"]
    B, Tq, Tk = case["B"], case["Tq"], case["Tk"]
    lengths = _lengths(case)

    def heads(*shape):
        # unit variance, a channel in 32 three times as large, as projections of hidden states have them
        x = torch.randn(*shape, generator=gen, device="cuda")
        x[..., ::32] *= 3.0
        return x

    s = {"case": case}
    if case["form"] == "ragged":
        rows = sum(n for n, _ in lengths)
        qkv = heads(rows, H + 2 * KV, D)
        qkv[:, H + KV:, ::32] /= 3.0
        s["qkv"] = qkv.to(dt)
        s["q"], s["k"], s["v"] = s["qkv"].split([H, KV, KV], dim=1)
        ends = [0]
        for n, _ in lengths:
            ends.append(ends[-1] + n)
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    else:
        s["q"], s["k"] = heads(B, Tq, H, D).to(dt), heads(B, Tk, KV, D).to(dt)
        s["v"] = torch.randn(B, Tk, KV, D, generator=gen, device="cuda").to(dt)
        if case["form"] != "dense":
            s["lengths"] = torch.tensor([n for _, n in lengths], dtype=torch.int32, device="cuda")
    if case["buckets"]:
        s["bias"] = torch.randn(case["buckets"], H, generator=gen, device="cuda").to(dt)
    if case["pass"] == "train":
        s["dout"] = torch.randn(s["q"].shape, generator=gen, device="cuda").to(dt)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2211_00839_amd as rcd

    case = s["case"]
    how = {"causal": case["causal"], "bias": s.get("bias"), "max_distance": case["distance"]}
    if case["form"] == "ragged":
        how.update(q_offsets=s["offsets"], k_offsets=s["offsets"], longest_q=case["Tq"], longest_k=case["Tk"])
    elif "lengths" in s:
        how.update(k_lengths=s["lengths"])
    if case["pass"] == "serve":
        return rcd.attention(s["q"], s["k"], s["v"], **how)
    out, saved = rcd.attention(s["q"], s["k"], s["v"], want_saved=True, **how)
    if case["form"] == "ragged":
        # the gradients go side by side, as the projection's backward pass takes them
        dqkv = torch.empty_like(s["qkv"])
        into = dqkv.split([case["heads"], case["kv_heads"], case["kv_heads"]], dim=1)
        grads = rcd.attention_backward(s["dout"], s["q"], s["k"], s["v"], out, saved, grads=into, **how)
        made = {"out": out, "dqkv": dqkv}
    else:
        grads = rcd.attention_backward(s["dout"], s["q"], s["k"], s["v"], out, saved, **how)
        made = {"out": out, "dq": grads.dq, "dk": grads.dk, "dv": grads.dv}
    if case["buckets"]:
        made["dbias"] = grads.dbias
    return made


def _borders(case):
    """The distances at which a bucket ends and the next begins, for one direction: 1, 2, .. up to half of its buckets, from
    there on in equal steps of the logarithm up to `distance`; in whole numbers, so that none is off by a rounding."""
    n = case["buckets"] if case["causal"] else case["buckets"] // 2
    exact, far = n // 2, case["distance"]
    steps = n - exact
    borders = list(range(1, exact + 1))
    r = exact
    for m in range(1, steps):
        while r ** steps < exact ** (steps - m) * far ** m:
            r += 1
        borders.append(r)
    return borders


def _buckets_plain(case, offset):
    """The bucket of each offset (key's position - query's): the number of borders that its size has reached; what follows the
    query has the second half of the buckets."""
    b = torch.zeros_like(offset)
    size = offset.abs()
    for border in _borders(case):
        b += size >= border
    if not case["causal"]:
        b += torch.where(offset > 0, case["buckets"] // 2, 0)
    return b


def _run_plain(s):
    case, f = s["case"], torch.float32
    H, KV, D, causal = case["heads"], case["kv_heads"], case["D"], case["causal"]
    G = H // KV
    train = case["pass"] == "train"
    q, k, v = s["q"], s["k"], s["v"]
    out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
    if train:
        dq, dk, dv = (torch.zeros(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        dbias = torch.zeros(case["buckets"], H, dtype=torch.float64, device=q.device)      # (long sums)
    scale = D ** -0.5
    at = 0
    grids = {}
    for b, (tq, tk) in enumerate(_lengths(case)):
        if case["form"] == "ragged":
            iq = ik = slice(at, at + tq)
            at += tq
        else:
            iq, ik = (b, slice(None)), (b, slice(0, tk))
        if (tq, tk) not in grids:
            if len(grids) > 8:
                grids.clear()
            offset = torch.arange(tk, device=q.device)[None, :] - torch.arange(tk - tq, tk, device=q.device)[:, None]
            grids[tq, tk] = (offset > 0 if causal else None, _buckets_plain(case, offset) if case["buckets"] else None)
        masked, bucket = grids[tq, tk]
        step = KV if H * tq * tk <= 2 ** 28 else 1        # heads of k and v taken at once
        for h in range(0, KV, step):
            hq, hk = slice(h * G, (h + step) * G), slice(h, h + step)
            qh = q[iq][:, hq].to(f).transpose(0, 1).reshape(step, G * tq, D)
            kh, vh = (t[ik][:, hk].to(f).transpose(0, 1).contiguous() for t in (k, v))
            score = (qh @ kh.transpose(1, 2).contiguous() * scale).reshape(step * G, tq, tk)
            if bucket is not None:
                score += s["bias"][:, hq].to(f).t()[:, bucket]
            if masked is not None:
                score.masked_fill_(masked, -math.inf)
            top = score.amax(2, keepdim=True)
            p = torch.exp(score.sub_(torch.where(top == -math.inf, 0.0, top)))
            total = p.sum(2, keepdim=True)
            p /= torch.where(total == 0, 1.0, total)        # (a query that sees no key gets zeros)
            p2 = p.reshape(step, G * tq, tk)
            o = (p2 @ vh).reshape(step * G, tq, D)
            out[iq][:, hq] = o.transpose(0, 1).to(out.dtype)
            if not train:
                continue
            do = s["dout"][iq][:, hq].to(f).transpose(0, 1)
            do2 = do.reshape(step, G * tq, D)
            dv[ik][:, hk] = (p2.transpose(1, 2).contiguous() @ do2).transpose(0, 1).to(dv.dtype)
            dp = (do2 @ vh.transpose(1, 2).contiguous()).reshape(step * G, tq, tk)
            ds = dp.sub_((do * o).sum(2, keepdim=True)).mul_(p)
            if bucket is not None:
                flat, each = bucket.reshape(-1), ds.reshape(step * G, -1)
                if flat.numel() <= 2 ** 18:
                    member = (flat[:, None] == torch.arange(case["buckets"], device=q.device)).to(torch.float64)
                    dbias[:, hq] += (each.to(torch.float64) @ member).t()
                else:
                    for c in range(case["buckets"]):
                        dbias[c, hq] += torch.where(flat == c, each, 0.0).sum(1, dtype=torch.float64)
            ds2 = ds.reshape(step, G * tq, tk)
            dq[iq][:, hq] = (ds2 @ kh * scale).reshape(step * G, tq, D).transpose(0, 1).to(dq.dtype)
            dk[ik][:, hk] = (ds2.transpose(1, 2).contiguous() @ qh * scale).transpose(0, 1).to(dk.dtype)
    if not train:
        return out
    made = {"out": out}
    if case["form"] == "ragged":
        made["dqkv"] = torch.cat([dq, dk, dv], dim=1)
    else:
        made.update(dq=dq, dk=dk, dv=dv)
    if case["buckets"]:
        made["dbias"] = dbias.to(s["bias"].dtype)
    return made


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------


def _reached(case, r):
    """The bucket of a distance r in its direction, from the definition: r itself below half of the buckets, then
    half + floor(steps ln(r / half) / ln(distance / half)), the last one at most; the floor by whole powers."""
    n = case["buckets"] // (1 if case["causal"] else 2)
    half = n // 2
    if r < half:
        return r
    best = 0
    while best < n - half - 1 and r ** (n - half) * half ** (best + 1) >= half ** (n - half) * case["distance"] ** (best + 1):
        best += 1
    return half + best


def exact(case, seed):
    s = prepare(case, seed)
    w = torch.float64
    H, per = case["heads"], case["heads"] // case["kv_heads"]
    lengths = _lengths(case)
    dev = s["q"].device
    packed = case["form"] == "ragged"
    q, k, v = (s[n].to(w) for n in ("q", "k", "v"))
    result = {"out": torch.zeros_like(q)}
    if case["pass"] == "train":
        g = s["dout"].to(w)
        result.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
        if case["buckets"]:
            result["dbias"] = torch.zeros(case["buckets"], H, dtype=w, device=dev)
    first = 0
    for b, (tq, tk) in enumerate(lengths):
        def part(t, n, h):
            return t[first:first + n, h] if packed else t[b, :n, h]

        span = torch.arange(-(tk - 1) - max(0, tk - tq), max(tk, tq) + tk, device=dev)       # every offset that there can be
        place = torch.arange(tk, device=dev) - (torch.arange(tq, device=dev) + (tk - tq)).unsqueeze(1)
        if case["buckets"]:
            far = case["distance"]
            small = torch.tensor([_reached(case, min(r, far)) for r in range(far + 1)], device=dev)
            which = small[span.abs().clamp(max=far)]
            if not case["causal"]:
                which = which + (span > 0) * (case["buckets"] // 2)
            which = which[place - span[0]]
        for h in range(H):
            qh, kh, vh = part(q, tq, h), part(k, tk, h // per), part(v, tk, h // per)
            z = torch.matmul(qh, kh.t()) / math.sqrt(case["D"])
            if case["buckets"]:
                z = z + s["bias"][:, h].to(w)[which]
            if case["causal"]:
                z = torch.where(place > 0, torch.full_like(z, -math.inf), z)
            p = torch.nan_to_num(torch.softmax(z, 1), nan=0.0) if case["causal"] and tq > tk else torch.softmax(z, 1)
            o = p @ vh
            part(result["out"], tq, h).copy_(o)
            if case["pass"] == "serve":
                continue
            gh = part(g, tq, h)
            part(result["dv"], tk, h // per).add_(p.t() @ gh)
            grad = p * (gh @ vh.t())
            grad = grad - p * grad.sum(1, keepdim=True)
            part(result["dq"], tq, h).copy_(grad @ kh / math.sqrt(case["D"]))
            part(result["dk"], tk, h // per).add_(grad.t() @ qh / math.sqrt(case["D"]))
            if case["buckets"]:
                result["dbias"][:, h].index_add_(0, which.reshape(-1), grad.reshape(-1))
        first += tq
    if case["pass"] == "serve":
        return result["out"]
    if packed:
        result = {"out": result["out"], "dqkv": torch.cat([result.pop(n) for n in ("dq", "dk", "dv")], 1), **{n: t for n, t in result.items() if n != "out"}}
    return result
