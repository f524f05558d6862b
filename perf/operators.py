"""The operators for a few tokens: what is measured, their plain forms, and their results in 64 bits.

* ``quantize``  weights to 4-bit codes with a scale (and a zero point) per group, and back to 16 bits
* ``gemv``      products of a few tokens with a 4-bit weight matrix
* ``moe``       a whole mixture-of-experts layer for a few tokens, 16-bit or 4-bit experts

4-bit codes are stored as the library stores them: a row of K weights has Kp / 2 bytes, Kp = K rounded up to a
multiple of 128.  Weight k = 128 b + 32 j + 8 t + i (j, t < 4, i < 8) is bits 4 n .. 4 n + 3, n = i / 2 + 4 (i % 2), of
the 32-bit little-endian word 16 b + 4 t + j of its row.  Scales and zero points are rows of Kp / group values.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- the cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # weights of a small projection, made when a model is loaded
        dict(name="quantize_small", op="quantize", N=1024, K=1024, group=128, zeros=False, src="bf16", dtype="bf16"),
        # a ragged matrix with zero points from a 32-bit checkpoint
        dict(name="quantize_ragged_zeros", op="quantize", N=5001, K=4100, group=32, zeros=True, src="fp32", dtype="fp16"),
        # a stack of experts
        dict(name="quantize_large", op="quantize", N=65536, K=4096, group=64, zeros=False, src="bf16", dtype="bf16"),
        # one token through a small projection: latency counts
        dict(name="gemv_small", op="gemv", T=1, N=1024, K=2048, group=128, zeros=False, dtype="bf16", out="bf16"),
        # one token through an ordinary square projection, zero points
        dict(name="gemv_token", op="gemv", T=1, N=4096, K=4096, group=64, zeros=True, dtype="fp16", out="fp16"),
        # a few tokens (speculative or small-batch decoding), ragged
        dict(name="gemv_ragged", op="gemv", T=5, N=5001, K=4100, group=32, zeros=True, dtype="bf16", out="fp32"),
        # one token through the largest projection: bandwidth counts
        dict(name="gemv_large", op="gemv", T=1, N=32768, K=16384, group=128, zeros=False, dtype="bf16", out="bf16"),
        # a batch of tokens through a wide projection
        dict(name="gemv_batch", op="gemv", T=24, N=16384, K=8192, group=128, zeros=False, dtype="bf16", out="bf16"),
        # one token, many small experts
        dict(name="moe_token", op="moe", T=1, H=2048, F=1024, E=64, top_k=8, shared=0, bits=16, group=0, zeros=False, dtype="bf16"),
        # a few tokens, ragged sizes, a shared expert
        dict(name="moe_ragged", op="moe", T=6, H=1416, F=1000, E=60, top_k=4, shared=1, bits=16, group=0, zeros=False, dtype="fp16"),
        # one token, few large 4-bit experts
        dict(name="moe_q4_token", op="moe", T=1, H=4096, F=8192, E=8, top_k=2, shared=0, bits=4, group=128, zeros=False, dtype="bf16"),
        # a decode batch that reaches nearly every expert
        dict(name="moe_batch", op="moe", T=64, H=4096, F=1536, E=64, top_k=6, shared=1, bits=16, group=0, zeros=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A size of [lo, hi]: multiples of 64, of 8, or any number."""
    n = _log(rng, lo, hi)
    m = rng.choice((64, 64, 64, 8, 1))
    n = max(lo, n - n % m)
    return n + 64 if n == 3072 else n


def draw(rng):
    most = max(work(c)["bytes"] + work(c)["flops"] / 200 for c in listed())
    while True:
        op = rng.choice(("quantize", "gemv", "gemv", "moe", "moe"))
        dtype, group, zeros = rng.choice(("bf16", "fp16")), rng.choice((32, 64, 128)), rng.random() < 0.5
        if op == "quantize":
            c = dict(op=op, N=_size(rng, 256, 65536), K=_size(rng, 256, 16384), group=group, zeros=zeros,
                     src=rng.choice((dtype, "fp32")), dtype=dtype)
        elif op == "gemv":
            c = dict(op=op, T=rng.choice((1, 1, _log(rng, 1, 32))), N=_size(rng, 256, 32768), K=_size(rng, 256, 16384),
                     group=group, zeros=zeros, dtype=dtype, out=rng.choice((dtype, dtype, "fp32")))
        else:
            bits = rng.choice((16, 4))
            E = _log(rng, 4, 256)
            c = dict(op=op, T=rng.choice((1, _log(rng, 1, 64))), H=_size(rng, 512, 7168), F=_size(rng, 256, 8192), E=E,
                     top_k=rng.randint(1, min(8, E)), shared=rng.choice((0, 0, 1)), bits=bits,
                     group=group if bits == 4 else 0, zeros=zeros if bits == 4 else False, dtype=dtype)
            if (c["E"] + c["shared"]) * c["H"] * c["F"] * bits > 3.2e10 or min(c["T"] * c["top_k"], E) * c["H"] * c["F"] > 2.5e9:
                continue
        w = work(c)
        if w["bytes"] + w["flops"] / 200 <= most:
            return c


def _groups(K, group):
    return (K + 127) // 128 * 128 // group


def work(case):
    c = case
    size = lambda d: 4 if d == "fp32" else 2  # noqa: E731
    if c["op"] == "quantize":  # the weights in, the values, scales and zero points out; the codes written and read
        held = c["N"] * (c["K"] / 2 + _groups(c["K"], c["group"]) * (3 if c["zeros"] else 2))
        return {"bytes": c["N"] * c["K"] * (size(c["src"]) + 2) + 2 * held, "flops": 4 * c["N"] * c["K"]}
    if c["op"] == "gemv":
        held = c["N"] * (c["K"] / 2 + _groups(c["K"], c["group"]) * (3 if c["zeros"] else 2))
        return {"bytes": held + c["T"] * (2 * c["K"] + size(c["out"]) * c["N"]), "flops": 2 * c["T"] * c["N"] * c["K"]}
    T, H, F, E, k, S = (c[n] for n in ("T", "H", "F", "E", "top_k", "shared"))
    taken = E * (1 - (1 - k / E) ** T) + S  # distinct experts, with tokens that choose independently
    if c["bits"] == 16:
        held = 3 * H * F * 2
    else:
        per = 3 if c["zeros"] else 2
        held = 3 * H * F / 2 + 2 * F * _groups(H, c["group"]) * per + H * _groups(F, c["group"]) * per
    return {"bytes": taken * held + E * H * 2 + T * (4 * H + 8 * k), "flops": T * ((k + S) * 6 * H * F + 2 * E * H)}


# ---- inputs ---------------------------------------------------------------------------------------------------
def _activations(T, K, dtype, g):
    """Normal values with a few channels that stand out, as the residual stream has them."""
    x = torch.randn(T, K, device=DEV, generator=g)
    loud = torch.rand(K, device=DEV, generator=g) < 0.01
    return (x * torch.where(loud, 8.0, 1.0)).to(dtype)


def _weights16(rows, K, dtype, g):
    return torch.empty(rows, K, device=DEV, dtype=dtype).normal_(0.0, K ** -0.5, generator=g)


def _weights4(rows, K, group, zeros, dtype, g):
    """Codes are uniform bytes; a scale is what a group of normal weights of deviation K^-1/2 has."""
    G = _groups(K, group)
    codes = torch.randint(0, 256, (rows, (K + 127) // 128 * 64), device=DEV, dtype=torch.uint8, generator=g)
    s = (torch.rand(rows, G, device=DEV, generator=g) * 0.2 + 0.3) * K ** -0.5
    z = torch.randint(5, 11, (rows, G), device=DEV, dtype=torch.uint8, generator=g) if zeros else None
    return {"codes": codes, "scales": s.to(dtype), "zeros": z, "rows": rows, "K": K, "group": group}


def _handle(m, dtype):
    """The library's view of a 4-bit matrix, kept beside its weights."""
    from paper_2609_16389_b200 import decode as D
    z = m["zeros"]
    return D.Q4(m["rows"], m["K"], m["group"], D.BF16 if dtype == torch.bfloat16 else D.FP16, m["codes"].data_ptr(),
                m["scales"].data_ptr(), 0 if z is None else z.data_ptr())


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "quantize":
        N, K = c["N"], c["K"]
        w = torch.empty(N, K, device=DEV, dtype=TYPES[c["src"]]).normal_(0.0, K ** -0.5, generator=g)
        s["w"] = w.mul_(torch.exp(0.5 * torch.randn(N, 1, device=DEV, generator=g)).to(w.dtype))  # rows differ in size
        m = _weights4(N, K, c["group"], c["zeros"], dt, g)  # room for the codes; what is in it is overwritten
        s["m"], s["values"] = m, torch.empty(N, K, device=DEV, dtype=dt)
        if own:
            s["q"] = _handle(m, dt)
    elif c["op"] == "gemv":
        s["m"] = _weights4(c["N"], c["K"], c["group"], c["zeros"], dt, g)
        s["x"] = _activations(c["T"], c["K"], dt, g)
        s["y"] = torch.empty(c["T"], c["N"], device=DEV, dtype=TYPES[c["out"]])
        if own:
            s["q"] = _handle(s["m"], dt)
    else:
        T, H, F, E, k, n = c["T"], c["H"], c["F"], c["E"], c["top_k"], c["E"] + c["shared"]
        s["x"] = _activations(T, H, dt, g)
        s["router"] = (1.5 * torch.randn(E, H, device=DEV, generator=g) * H ** -0.5).to(dt)
        for name, rows, K in (("gate", F, H), ("up", F, H), ("down", H, F)):
            s[name] = (_weights16(n * rows, K, dt, g) if c["bits"] == 16
                       else _weights4(n * rows, K, c["group"], c["zeros"], dt, g))
        s["y"] = torch.empty(T, H, device=DEV, dtype=dt)
        s["index"] = torch.empty(T, k, device=DEV, dtype=torch.int32)
        s["weight"] = torch.empty(T, k, device=DEV)
        if own:
            from paper_2609_16389_b200 import decode as D
            s["plan"] = D.MoePlan(D.MoeDesc(H, F, E, c["shared"], k, T, D.BF16 if c["dtype"] == "bf16" else D.FP16,
                                            c["group"], 1, 1.0))
            mats = []
            for name, rows, K in (("gate", F, H), ("up", F, H), ("down", H, F)):
                m = s[name]
                mats.append(D.MoeMatrix(m.data_ptr(), K, rows, 0, 0) if c["bits"] == 16 else
                            D.MoeMatrix(m["codes"].data_ptr(), 0, rows, m["scales"].data_ptr(),
                                        0 if m["zeros"] is None else m["zeros"].data_ptr()))
            s["weights"] = D.MoeWeights(s["router"].data_ptr(), H, *mats)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "quantize":
        return _plain_quantize(s["w"], c["group"], c["zeros"], TYPES[c["dtype"]])
    if c["op"] == "gemv":
        m = s["m"]
        w = _plain_values(m["codes"], m["scales"], m["zeros"], c["K"], c["group"])
        return {"y": (s["x"].float() @ w.t()).to(TYPES[c["out"]])}
    return _plain_moe(s, c)


def _run_own(s):
    from paper_2609_16389_b200 import decode as D
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "quantize":
        w, v, q = s["w"], s["values"], s["q"]
        q.quantize(w.data_ptr(), c["K"], {"bf16": D.BF16, "fp16": D.FP16, "fp32": D.FP32}[c["src"]], stream)
        q.dequantize(v.data_ptr(), c["K"], D.BF16 if c["dtype"] == "bf16" else D.FP16, stream)
        out = {"values": v, "scales": s["m"]["scales"]}
        return {**out, "zeros": s["m"]["zeros"]} if c["zeros"] else out
    if c["op"] == "gemv":
        y = s["y"]
        s["q"].gemv(c["T"], s["x"].data_ptr(), c["K"], y.data_ptr(), c["N"],
                    {"bf16": D.BF16, "fp16": D.FP16, "fp32": D.FP32}[c["out"]], 1.0, 0.0, stream)
        return {"y": y}
    s["plan"].run(s["weights"], c["T"], s["x"].data_ptr(), c["H"], s["y"].data_ptr(), c["H"], s["index"].data_ptr(),
                  s["weight"].data_ptr(), stream)
    return {"y": s["y"], "index": s["index"], "weight": s["weight"]}


def _plain_quantize(w, group, zeros, dtype):
    """Divisions are by tensors: a division by a Python number may be computed as a product with its reciprocal."""
    N, K = w.shape
    Kp = (K + 127) // 128 * 128
    v = torch.zeros(N, Kp, device=w.device)
    v[:, :K] = w
    v = v.view(N, Kp // group, group)
    if zeros:
        lo, hi = v.amin(2).clamp(max=0.0), v.amax(2).clamp(min=0.0)
        s16 = ((hi - lo) / torch.full_like(lo, 15.0)).to(dtype)
        s = torch.where(s16 > 0, s16.float(), 1.0)
        z = torch.where(s16 > 0, torch.round(-lo / s).clamp(0, 15), 8.0)
        q = (torch.round(v / s[:, :, None]) + z[:, :, None]).clamp(0, 15)
    else:
        top = v.abs().amax(2)
        s16 = (top / torch.full_like(top, 7.0)).to(dtype)
        s = torch.where(s16 > 0, s16.float(), 1.0)
        z = torch.full_like(s, 8.0)
        q = torch.round(v / s[:, :, None]).clamp(-8, 7) + 8.0
    q = torch.where((s16 > 0)[:, :, None], q, z[:, :, None])
    values = ((q - z[:, :, None]) * s16.float()[:, :, None]).view(N, Kp)[:, :K].to(dtype)
    out = {"values": values, "scales": s16}
    return {**out, "zeros": z.to(torch.uint8)} if zeros else out


def _plain_values(codes, scales, zeros, K, group):
    """fp32 values of rows of codes (leading dimensions are kept)."""
    lead, Kp = codes.shape[:-1], 2 * codes.shape[-1]
    n = torch.stack((codes & 15, codes >> 4), -1).view(*lead, Kp // 128, 4, 4, 2, 4)  # block, t, j, i % 2, i / 2
    d = len(lead)
    q = n.permute(*range(d), d, d + 2, d + 1, d + 4, d + 3).reshape(*lead, Kp // group, group).float()
    z = 8.0 if zeros is None else zeros.float()[..., None]
    return ((q - z) * scales.float()[..., None]).view(*lead, Kp)[..., :K]


def _plain_moe(s, c):
    T, H, F, E, k, S = (c[n] for n in ("T", "H", "F", "E", "top_k", "shared"))
    x = s["x"].float()
    p = torch.softmax(x @ s["router"].float().t(), 1)
    weight, index = torch.sort(p, dim=1, descending=True, stable=True)  # equal ones: the lowest index first
    weight, index = weight[:, :k], index[:, :k]
    weight = weight / weight.sum(1, keepdim=True)

    def of(name, rows, K, at=None):
        """fp32 weights of the experts `at` (all of them if None), [experts, rows, K]."""
        take = (lambda t: t.view(E + S, rows, -1)) if at is None else (lambda t: t.view(E + S, rows, -1)[at])
        if c["bits"] == 16:
            return take(s[name]).float()
        m = s[name]
        return _plain_values(take(m["codes"]), take(m["scales"]), None if m["zeros"] is None else take(m["zeros"]), K, c["group"])

    if T * (k + S) < E + S:  # the taken experts' weights, once for every token that takes them
        at = torch.cat((index, torch.arange(E, E + S, device=DEV).expand(T, S)), 1).reshape(-1)
        wt = torch.cat((weight, torch.ones(T, S, device=DEV)), 1).reshape(-1, 1)
        rows = x.repeat_interleave(k + S, 0)[:, :, None]
        h = torch.nn.functional.silu(torch.bmm(of("gate", F, H, at), rows)) * torch.bmm(of("up", F, H, at), rows)
        y = (torch.bmm(of("down", H, F, at), h)[:, :, 0] * wt).view(T, k + S, H).sum(1)
    else:                    # every expert on every token
        wt = torch.cat((torch.zeros(T, E, device=DEV).scatter(1, index, weight), torch.ones(T, S, device=DEV)), 1)
        h = torch.nn.functional.silu(x @ of("gate", F, H).transpose(1, 2)) * (x @ of("up", F, H).transpose(1, 2))
        y = torch.bmm(h * wt.t()[:, :, None], of("down", H, F).transpose(1, 2)).sum(0)
    return {"y": y.to(s["y"].dtype), "index": index.to(torch.int32), "weight": weight}


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _values64(m, rows):
    """64-bit values of the rows `rows` (a slice) of a 4-bit matrix, weight by weight from the layout's definition."""
    K, group = m["K"], m["group"]
    at = torch.arange(K, device=DEV)
    b, r = at // 128, at % 128
    i = r % 8
    n = i // 2 + 4 * (i % 2)
    byte = 64 * b + 16 * (r % 32 // 8) + 4 * (r // 32) + n // 2
    q = (m["codes"][rows][:, byte].to(torch.int32) >> (4 * (n % 2))) & 15
    z = 8 if m["zeros"] is None else m["zeros"][rows][:, at // group].to(torch.int32)
    return (q - z).double() * m["scales"][rows].double()[:, at // group]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "quantize":
        w, group, dt = s["w"].double(), c["group"], TYPES[c["dtype"]]
        values, scales, zs = torch.empty_like(w), [], []
        for lo in range(0, _groups(c["K"], group) * group, group):
            part = w[:, lo:lo + group]
            if part.shape[1] == 0:  # a group that is all padding
                part = torch.zeros_like(w[:, :1])
            if c["zeros"]:
                a, b = part.min(1, keepdim=True)[0].clamp(max=0), part.max(1, keepdim=True)[0].clamp(min=0)
                sc = ((b - a) / 15).float().to(dt).double()
                d = torch.where(sc > 0, sc, torch.ones_like(sc))
                z = torch.where(sc > 0, (-a / d).round().clamp(0, 15), torch.full_like(sc, 8))
                q = ((part / d).round() + z).clamp(0, 15) - z
            else:
                sc = (part.abs().max(1, keepdim=True)[0] / 7).float().to(dt).double()
                d = torch.where(sc > 0, sc, torch.ones_like(sc))
                z = torch.full_like(sc, 8)
                q = (part / d).round().clamp(-8, 7)
            if lo < c["K"]:
                values[:, lo:lo + group] = q * sc
            scales.append(sc)
            zs.append(z)
        out = {"values": values, "scales": torch.cat(scales, 1)}
        return {**out, "zeros": None} if c["zeros"] else out
    x = s["x"].double()
    if c["op"] == "gemv":
        y = torch.empty(c["T"], c["N"], device=DEV, dtype=torch.float64)
        for lo in range(0, c["N"], 2048):
            y[:, lo:lo + 2048] = x @ _values64(s["m"], slice(lo, lo + 2048)).t()
        return {"y": y}
    T, H, F, E, k = (c[n] for n in ("T", "H", "F", "E", "top_k"))
    e = torch.exp(x @ s["router"].double().t())
    y, weight = torch.zeros(T, H, device=DEV, dtype=torch.float64), torch.empty(T, k, device=DEV, dtype=torch.float64)
    w64 = lambda name, at, rows: (s[name][at * rows:(at + 1) * rows].double() if c["bits"] == 16  # noqa: E731
                                  else _values64(s[name], slice(at * rows, (at + 1) * rows)))
    part = torch.zeros(T, E + c["shared"], device=DEV, dtype=torch.float64)
    part[:, E:] = 1
    for t in range(T):
        best = torch.topk(e[t], k)
        weight[t] = best.values / best.values.sum()
        part[t, best.indices] = weight[t]
    for at in range(E + c["shared"]):
        toks = part[:, at].nonzero()[:, 0]
        if len(toks):
            g = x[toks] @ w64("gate", at, F).t()
            h = g / (1 + torch.exp(-g)) * (x[toks] @ w64("up", at, F).t())
            y[toks] += part[toks, at][:, None] * (h @ w64("down", at, H).t())
    return {"y": y, "index": None, "weight": weight}
