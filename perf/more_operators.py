"""Products whose epilogue is the operator: what is measured, their plain forms, and their results in 64 bits.

* ``ffn``  a gated feed-forward block y = (act(x Wg^T) * (x Wu^T)) Wd^T, and with ``train`` its backward pass
* ``ce``   softmax cross entropy of a head x W^T over a vocabulary, and with ``train`` its gradients
* ``i8``   activations to 8-bit integers with a scale per token, and their product with 8-bit weights with a scale per channel

gate and up are the two halves of one matrix of 2 * F rows.  Targets outside 0 .. V - 1 are ignored: loss 0, no gradient.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = ("silu", "gelu", "gelu_tanh")


# ---- the cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token through a block: latency and the weights' bandwidth count
        dict(name="ffn_token", op="ffn", train=False, T=1, H=4096, F=10240, act="silu", dtype="bf16"),
        # a decode batch, ragged sizes
        dict(name="ffn_decode_ragged", op="ffn", train=False, T=24, H=2056, F=5500, act="gelu_tanh", dtype="fp16"),
        # a prompt
        dict(name="ffn_prompt", op="ffn", train=False, T=2048, H=4096, F=12288, act="silu", dtype="bf16"),
        # a small model's training step
        dict(name="ffn_train_small", op="ffn", train=True, T=512, H=1024, F=2816, act="silu", dtype="bf16"),
        # ragged sizes, the exact Gaussian gate
        dict(name="ffn_train_ragged", op="ffn", train=True, T=1001, H=1544, F=4100, act="gelu", dtype="fp16"),
        # a large model's training step
        dict(name="ffn_train_large", op="ffn", train=True, T=8192, H=4096, F=12288, act="silu", dtype="bf16"),
        # scores of a few answers (no gradient) over an odd vocabulary
        dict(name="ce_score", op="ce", train=False, T=64, H=2048, V=50257, smoothing=0.0, dtype="bf16"),
        # a small model's training step, smoothed labels
        dict(name="ce_train_ragged", op="ce", train=True, T=1000, H=1024, V=32001, smoothing=0.1, dtype="fp16"),
        # a large vocabulary's training step
        dict(name="ce_train_large", op="ce", train=True, T=8192, H=4096, V=128000, smoothing=0.0, dtype="bf16"),
        # one token through a projection: latency and the weights' bandwidth count
        dict(name="i8_token", op="i8", T=1, N=8192, K=8192, dtype="bf16", out="bf16"),
        # a few tokens, ragged sizes, 32-bit results
        dict(name="i8_ragged", op="i8", T=37, N=5001, K=4100, dtype="fp16", out="fp32"),
        # a prompt through a wide projection
        dict(name="i8_prompt", op="i8", T=4096, N=12288, K=4096, dtype="bf16", out="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, multiples=(64, 64, 64, 8, 1)):
    """A size of [lo, hi]: multiples of 64, of 8, or any number."""
    n = _log(rng, lo, hi)
    return max(lo, n - n % rng.choice(multiples))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("ffn", "ffn", "ce", "ce", "i8"))
        dtype, train = rng.choice(("bf16", "fp16")), rng.random() < 0.6
        T = rng.choice((_log(rng, 1, 64), _size(rng, 64, 8192, (64, 1))))
        if op == "ffn":
            c = dict(op=op, train=train, T=T, H=_size(rng, 256, 8192, (64, 64, 8)), F=_size(rng, 256, 28672, (64, 64, 8, 2)),
                     act=rng.choice(ACTS), dtype=dtype)
        elif op == "ce":
            c = dict(op=op, train=train, T=T, H=_size(rng, 256, 8192, (64, 64, 8)), V=_size(rng, 1000, 131072, (64, 8, 1)),
                     smoothing=rng.choice((0.0, 0.0, 0.1)), dtype=dtype)
        else:
            c = dict(op=op, T=T, N=_size(rng, 256, 32768), K=_size(rng, 256, 16384), dtype=dtype, out=rng.choice((dtype, dtype, "fp32")))
        if _cost(c) <= most:
            return c


def _cost(c):
    w = work(c)
    return w["bytes"] + w["flops"] / 200


def work(case):
    c, T = case, case["T"]
    if c["op"] == "ffn":
        H, F = c["H"], c["F"]
        if not c["train"]:
            return {"bytes": 2 * (3 * H * F + 2 * T * H), "flops": 6 * T * H * F}
        # x, dy and the weights in, y, dx and the weights' gradients out
        return {"bytes": 2 * (6 * H * F + 4 * T * H), "flops": 18 * T * H * F}
    if c["op"] == "ce":
        H, V = c["H"], c["V"]
        if not c["train"]:
            return {"bytes": 2 * (V * H + T * H) + 16 * T, "flops": 2 * T * H * V}
        return {"bytes": 4 * (V * H + T * H) + 20 * T, "flops": 6 * T * H * V}
    N, K = c["N"], c["K"]
    return {"bytes": N * K + 4 * N + 2 * T * K + (4 if c["out"] == "fp32" else 2) * T * N + 4 * T, "flops": 2 * T * N * K}


# ---- inputs ---------------------------------------------------------------------------------------------------
def _normal(rows, cols, deviation, dtype, g):
    return torch.empty(rows, cols, device=DEV, dtype=dtype).normal_(0.0, deviation, generator=g)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, T = TYPES[c["dtype"]], c["T"]
    s = {"case": c}
    if c["op"] == "ffn":
        H, F = c["H"], c["F"]
        s["x"] = _normal(T, H, 1.0, dt, g)
        s["gate_up"] = _normal(2 * F, H, 1.5 * H ** -0.5, dt, g)
        s["down"] = _normal(H, F, F ** -0.5, dt, g)
        s["y"] = torch.empty(T, H, device=DEV, dtype=dt)
        if c["train"]:
            s["dy"] = _normal(T, H, 2.0 ** -6, dt, g)
            s["dx"], s["dgate_up"], s["ddown"] = (torch.empty_like(s[n]) for n in ("x", "gate_up", "down"))
        if own:
            from paper_2609_16389_b200 import fused as E
            t = E.BF16 if c["dtype"] == "bf16" else E.FP16
            act = {"silu": E.SILU, "gelu": E.GELU, "gelu_tanh": E.GELU_TANH}[c["act"]]
            s["plan"] = E.FfnPlan(E.FfnDesc(T, H, F, t, act, training=int(c["train"]), grad_dtype=t))
            s["saved"] = torch.empty(s["plan"].saved_bytes(), device=DEV, dtype=torch.uint8)
    elif c["op"] == "ce":
        H, V = c["H"], c["V"]
        s["x"] = _normal(T, H, 1.0, dt, g)
        s["w"] = _normal(V, H, 2.0 * H ** -0.5, dt, g)
        target = torch.randint(0, V, (T,), device=DEV, generator=g)
        # a few rows are padding; the first never is, so that something is learned
        s["target"] = torch.where((torch.rand(T, device=DEV, generator=g) < 0.05) & (torch.arange(T, device=DEV) > 0), -100, target)
        s["loss"], s["lse"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        if c["train"]:
            # a weighted mean; half-precision training scales its loss
            s["dloss"] = (0.5 + torch.rand(T, device=DEV, generator=g)) * ((1024.0 if c["dtype"] == "fp16" else 1.0) / T)
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        if own:
            from paper_2609_16389_b200 import fused as E
            t = E.BF16 if c["dtype"] == "bf16" else E.FP16
            s["plan"] = E.CePlan(E.CeDesc(T, H, V, t, training=int(c["train"]), grad_dtype=t, label_smoothing=c["smoothing"]))
            s["saved"] = torch.empty(s["plan"].saved_bytes(), device=DEV, dtype=torch.uint8)
    else:
        N, K = c["N"], c["K"]
        x = torch.randn(T, K, device=DEV, generator=g)
        loud = torch.rand(K, device=DEV, generator=g) < 0.01  # a few channels that stand out, as the residual stream has them
        s["x"] = (x * torch.where(loud, 8.0, 1.0)).to(dt)
        ld = (K + 15) // 16 * 16  # rows of codes start on 16 bytes
        s["w"] = torch.randint(-127, 128, (N, ld), device=DEV, dtype=torch.int8, generator=g)
        s["ws"] = (torch.rand(N, device=DEV, generator=g) * 0.4 + 0.8) * (K ** -0.5 / 64)
        s["codes"] = torch.empty(T, ld, device=DEV, dtype=torch.int8)
        s["scales"] = torch.empty(T, device=DEV)
        s["y"] = torch.empty(T, N, device=DEV, dtype=TYPES[c["out"]])
        if own:
            from paper_2609_16389_b200 import fused as E
            s["qx"] = E.I8(T, K, ld, s["codes"].data_ptr(), s["scales"].data_ptr())
            s["qw"] = E.I8(N, K, ld, s["w"].data_ptr(), s["ws"].data_ptr())
    return s


# ---- one pass -------------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "ffn":
        return _plain_ffn(s, c)
    if c["op"] == "ce":
        return _plain_ce(s, c)
    x = s["x"].float()
    top = x.abs().amax(1)
    scale = top / torch.full_like(top, 127.0)  # a division by a Python number may be a product with its reciprocal
    safe = torch.where(scale > 0, scale, 1.0)
    codes = torch.where((scale > 0)[:, None], torch.round(x / safe[:, None]).clamp(-127, 127), 0.0)
    sums = codes.double() @ s["w"][:, :c["K"]].double().t()  # 32 bits do not hold these sums
    return {"y": (sums.float() * scale[:, None] * s["ws"][None, :]).to(TYPES[c["out"]]), "scales": scale}


def _run_own(s):
    from paper_2609_16389_b200 import fused as E
    c, stream = s["case"], torch.cuda.current_stream().cuda_stream
    p = lambda name: s[name].data_ptr()  # noqa: E731
    if c["op"] == "ffn":
        plan = s["plan"]
        if not c["train"]:
            plan.forward(p("x"), p("gate_up"), p("down"), p("y"), stream=stream)
            return {"y": s["y"]}
        plan.forward(p("x"), p("gate_up"), p("down"), p("y"), p("saved"), stream=stream)
        plan.backward(p("x"), p("gate_up"), p("down"), p("saved"), p("dy"), p("dx"), p("dgate_up"), p("ddown"), stream=stream)
        return {n: s[n] for n in ("y", "dx", "dgate_up", "ddown")}
    if c["op"] == "ce":
        plan = s["plan"]
        if not c["train"]:
            plan.forward(p("x"), p("w"), p("target"), p("loss"), p("lse"), stream=stream)
            return {"loss": s["loss"], "lse": s["lse"]}
        plan.forward(p("x"), p("w"), p("target"), p("loss"), p("lse"), p("saved"), stream)
        plan.backward(p("x"), p("w"), p("target"), p("lse"), p("dloss"), p("saved"), p("dx"), p("dw"), stream=stream)
        return {n: s[n] for n in ("loss", "lse", "dx", "dw")}
    s["qx"].quantize(p("x"), c["K"], E.BF16 if c["dtype"] == "bf16" else E.FP16, stream)
    s["qw"].gemm(s["qx"], p("y"), c["N"], {"bf16": E.BF16, "fp16": E.FP16, "fp32": E.FP32}[c["out"]], stream=stream)
    return {"y": s["y"], "scales": s["scales"]}


def _plain_act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * 2.0 ** -0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    a, b = (2.0 / math.pi) ** 0.5, 0.044715
    t = torch.tanh(a * (g + b * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * a * (1.0 + 3.0 * b * g * g)


def _plain_ffn(s, c):
    dt, F = TYPES[c["dtype"]], c["F"]
    x, gu, down = s["x"].float(), s["gate_up"].float(), s["down"].float()
    z = x @ gu.t()
    g, u = z[:, :F], z[:, F:]
    a, slope = _plain_act(g, c["act"])
    h = a * u
    out = {"y": (h @ down.t()).to(dt)}
    if c["train"]:
        dy = s["dy"].float()
        dh = dy @ down
        dz = torch.cat((dh * u * slope, dh * a), 1)
        out.update(dx=(dz @ gu).to(dt), dgate_up=(dz.t() @ x).to(dt), ddown=(dy.t() @ h).to(dt))
    return out


def _plain_ce(s, c):
    dt, V, eps = TYPES[c["dtype"]], c["V"], c["smoothing"]
    x, w, target = s["x"].float(), s["w"].float(), s["target"]
    logits = x @ w.t()
    top = logits.amax(1, keepdim=True)
    lse = torch.log(torch.exp(logits - top).sum(1)) + top[:, 0]
    taken = (target >= 0) & (target < V)
    at = torch.where(taken, target, 0)
    loss = lse - (1.0 - eps) * logits.gather(1, at[:, None])[:, 0]
    if eps:
        loss = loss - eps * logits.double().mean(1).float()
    out = {"loss": torch.where(taken, loss, 0.0), "lse": lse}
    if c["train"]:
        d = logits.sub_(lse[:, None]).exp_()
        if eps:
            d = d.sub_(eps / V)
        d.scatter_add_(1, at[:, None], torch.full_like(lse, eps - 1.0)[:, None])
        d.mul_(torch.where(taken, s["dloss"], 0.0)[:, None])
        out.update(dx=(d @ w).to(dt), dw=(d.t() @ x).to(dt))
    return out


# ---- the definition in 64 bits --------------------------------------------------------------------------------
def _exact_act(z, act):
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    x, T = s["x"].double(), c["T"]
    if c["op"] == "i8":
        y, scales = torch.empty(T, c["N"], device=DEV, dtype=torch.float64), (x.abs().max(1)[0] / 127).float().double()
        codes = torch.round(x / scales[:, None]).clamp(-127, 127)
        for lo in range(0, c["N"], 4096):
            rows = slice(lo, lo + 4096)
            y[:, rows] = (codes * scales[:, None]) @ (s["w"][rows, :c["K"]].double() * s["ws"][rows].double()[:, None]).t()
        return {"y": y, "scales": scales}
    if c["op"] == "ffn":
        H, F = c["H"], c["F"]
        y = torch.zeros(T, H, device=DEV, dtype=torch.float64)
        if c["train"]:
            dy, dx = s["dy"].double(), torch.zeros(T, H, device=DEV, dtype=torch.float64)
            dgu = torch.empty(2 * F, H, device=DEV, dtype=torch.float64)
            ddown = torch.empty(H, F, device=DEV, dtype=torch.float64)
        for lo in range(0, F, 4096):  # a block of inner channels at a time
            hi = min(lo + 4096, F)
            wg, wu, wd = s["gate_up"][lo:hi].double(), s["gate_up"][F + lo:F + hi].double(), s["down"][:, lo:hi].double()
            gate = (x @ wg.t()).requires_grad_(c["train"])
            up, a = x @ wu.t(), _exact_act(gate, c["act"])
            h = a.detach() * up
            y += h @ wd.t()
            if c["train"]:
                dh = dy @ wd
                dgate, = torch.autograd.grad(a, gate, dh * up)
                dup = dh * a.detach()
                dx += dgate @ wg + dup @ wu
                dgu[lo:hi], dgu[F + lo:F + hi], ddown[:, lo:hi] = dgate.t() @ x, dup.t() @ x, dy.t() @ h
        return {"y": y, "dx": dx, "dgate_up": dgu, "ddown": ddown} if c["train"] else {"y": y}
    V, eps, target, step = c["V"], c["smoothing"], s["target"], 8192
    lse = torch.full((T,), -math.inf, device=DEV, dtype=torch.float64)
    mean, hit = torch.zeros_like(lse), torch.zeros_like(lse)
    taken = ((target >= 0) & (target < V)).double()

    def onehot(lo, hi):
        return (target[:, None] == torch.arange(lo, hi, device=DEV)[None, :]).double()

    for lo in range(0, V, step):
        hi = min(lo + step, V)
        z = x @ s["w"][lo:hi].double().t()
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        mean += z.sum(1) / V
        hit += (z * onehot(lo, hi)).sum(1)
    out = {"loss": taken * (lse - (1 - eps) * hit - eps * mean), "lse": lse}
    if c["train"]:
        weight, dx = (taken * s["dloss"].double())[:, None], torch.zeros_like(x)
        dw = torch.empty(V, c["H"], device=DEV, dtype=torch.float64)
        for lo in range(0, V, step):
            hi = min(lo + step, V)
            w = s["w"][lo:hi].double()
            d = weight * (torch.exp(x @ w.t() - lse[:, None]) - (1 - eps) * onehot(lo, hi) - eps / V)
            dx += d @ w
            dw[lo:hi] = d.t() @ x
        out.update(dx=dx, dw=dw)
    return out
