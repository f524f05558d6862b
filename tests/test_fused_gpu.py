"""Products with an operator in their epilogue against 64-bit results with counted roundings (fused_reference.py)."""
import pytest
import torch

import fused_reference as R
from paper_2609_16389_b200 import fused as E

pytestmark = pytest.mark.gpu

DT = {"bf16": (torch.bfloat16, E.BF16), "fp16": (torch.float16, E.FP16)}
ACT = {"silu": E.SILU, "gelu": E.GELU, "gelu_tanh": E.GELU_TANH}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def strided(rows, cols, dtype, g, ld=0, scale=1.0, fill=None):
    """A rows x cols view of a matrix with leading dimension ld, whose gap holds NaN (or `fill`), and so do two rows behind it."""
    ld = ld or cols
    whole = torch.full((rows + 2, ld), float("nan") if fill is None else fill, device="cuda", dtype=dtype)
    view = whole[:rows, :cols]
    if g is not None:
        view.copy_(torch.randn(rows, cols, device="cuda", generator=g) * scale)
    return whole, view


def stream():
    return torch.cuda.current_stream().cuda_stream


class Ffn:
    def __init__(self, T, H, F, dtype, act, train, grad="same", lds=(0, 0, 0, 0), seed=0):
        dt, code = DT[dtype]
        g = gen(seed)
        ldx, ldy, ldg, ldd = lds
        self.x0, self.x = strided(T, H, dt, g, ldx)
        self.gu0, self.gate_up = strided(2 * F, H, dt, g, ldg, 1.5 * H ** -0.5)
        self.d0, self.down = strided(H, F, dt, g, ldd, F ** -0.5)
        self.y0, self.y = strided(T, H, dt, None, ldy, fill=7.0)
        self.dy0, self.dy = strided(T, H, dt, g, ldy, 2.0 ** -6)
        gt, gcode = (torch.float32, E.FP32) if grad == "fp32" else (dt, code)
        self.dx0, self.dx = strided(T, H, dt, None, ldx, fill=7.0)
        self.dgu0, self.dgate_up = strided(2 * F, H, gt, None, ldg, fill=7.0)
        self.dd0, self.ddown = strided(H, F, gt, None, ldd, fill=7.0)
        self.act = act
        self.plan = E.FfnPlan(E.FfnDesc(T, H, F, code, ACT[act], int(train), gcode, ldx, ldy, ldg, ldd))
        self.saved = torch.full((self.plan.saved_bytes() + 256,), 255, device="cuda", dtype=torch.uint8)   # NaN, if it were read

    def forward(self, saved=True):
        self.plan.forward(self.x0.data_ptr(), self.gu0.data_ptr(), self.d0.data_ptr(), self.y0.data_ptr(), self.saved.data_ptr() if saved else 0,
                          stream())

    def backward(self, accumulate=0, dx=True, dgu=True, dd=True):
        self.plan.backward(self.x0.data_ptr(), self.gu0.data_ptr(), self.d0.data_ptr(), self.saved.data_ptr(), self.dy0.data_ptr(),
                           self.dx0.data_ptr() if dx else 0, self.dgu0.data_ptr() if dgu else 0, self.dd0.data_ptr() if dd else 0, accumulate, stream())

    def want(self, train):
        return R.ffn(self.x, self.gate_up, self.down, self.act, self.dy if train else None)

    def check_forward(self, want):
        self.plan.check()
        R.check(self.y, want["y"], "y")
        assert (self.saved[self.plan.saved_bytes():] == 255).all() and (self.y0[self.y.shape[0]:] == 7.0).all()

    def check_backward(self, want):
        self.plan.check()
        R.check(self.dx, want["dx"], "dx")
        for name, got in (("dgate_up", self.dgate_up), ("ddown", self.ddown)):
            R.check(got, R.rounded(want[name], got.dtype), name)
        for whole, view in ((self.dx0, self.dx), (self.dgu0, self.dgate_up), (self.dd0, self.ddown)):
            assert (whole[view.shape[0]:] == 7.0).all()

    def gaps_untouched(self, train):
        for whole, view in ((self.y0, self.y),) + (((self.dx0, self.dx), (self.dgu0, self.dgate_up), (self.dd0, self.ddown)) if train else ()):
            assert (whole[:, view.shape[1]:] == 7.0).all() and (whole[view.shape[0]:] == 7.0).all()


FFN_SIZES = [(1, 64, 64), (1, 264, 8), (2, 8, 1), (2, 1, 3), (140, 1, 1), (70, 37, 44), (3, 4104, 40), (70, 2064, 200), (1, 72, 4100), (5, 72, 35), (33, 136, 200), (64, 520, 1100), (128, 264, 2400), (129, 264, 136), (200, 136, 72),
             (300, 1032, 516), (513, 72, 1025)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,H,F", FFN_SIZES)
def test_ffn_forward(T, H, F, dtype):
    for act in ACT:
        f = Ffn(T, H, F, dtype, act, False, seed=T + F)
        f.forward(saved=False)
        f.check_forward(f.want(False))


@pytest.mark.parametrize("T,H,F,dtype,act,grad", [
    (1, 64, 64, "bf16", "silu", "same"), (3, 72, 40, "fp16", "gelu", "fp32"), (128, 264, 200, "bf16", "gelu_tanh", "fp32"),
    (129, 264, 136, "fp16", "silu", "same"), (257, 520, 516, "bf16", "gelu", "same"), (300, 136, 1030, "fp16", "gelu_tanh", "same"),
    (511, 1032, 257, "bf16", "silu", "fp32"), (140, 72, 260, "bf16", "gelu", "same"), (140, 72, 262, "bf16", "silu", "same"), (7, 1, 1, "fp16", "silu", "same"), (1000, 256, 2304, "bf16", "silu", "same"), (2, 8, 1, "bf16", "gelu", "same")])
def test_ffn_training(T, H, F, dtype, act, grad):
    f = Ffn(T, H, F, dtype, act, True, grad, seed=T)
    f.forward()
    f.backward()
    want = f.want(True)
    f.check_forward(want)
    f.check_backward(want)


@pytest.mark.parametrize("T,H,F,lds", [
    (7, 65, 35, (0, 0, 0, 0)),                 # odd rows: every matrix goes through an aligned copy
    (130, 65, 35, (0, 0, 0, 0)),
    (7, 64, 40, (72, 80, 96, 64)),             # gaps
    (150, 64, 40, (67, 80, 65, 41)),           # some matrices aligned, some not
    (150, 72, 48, (80, 73, 80, 56)),
    (150, 65, 35, (72, 80, 72, 40))])          # rows that end inside a 16-byte piece, with a gap behind them
def test_ffn_strides(T, H, F, lds):
    f = Ffn(T, H, F, "bf16", "silu", True, lds=lds, seed=3)
    f.forward()
    f.backward()
    want = f.want(True)
    f.check_forward(want)
    f.check_backward(want)
    f.gaps_untouched(True)


@pytest.mark.parametrize("T", [1, 200])
def test_ffn_accumulates_and_leaves_out(T):
    f = Ffn(T, 136, 72, "bf16", "silu", True, "fp32", seed=5)
    f.forward()
    f.backward()
    first = [t.clone() for t in (f.dx, f.dgate_up, f.ddown)]
    f.backward(accumulate=1)
    assert torch.equal(f.dx, first[0])         # the gradient of x is never accumulated
    assert torch.equal(f.dgate_up, 2 * first[1]) and torch.equal(f.ddown, 2 * first[2])
    for left_out in range(3):
        for t in (f.dx, f.dgate_up, f.ddown):
            t.fill_(5.0)
        f.backward(0, left_out != 0, left_out != 1, left_out != 2)
        for i, t in enumerate((f.dx, f.dgate_up, f.ddown)):
            assert torch.equal(t, torch.full_like(t, 5.0) if i == left_out else first[i])


def test_ffn_gradients_against_differences():
    """The gradients, through a scalar loss, against differences of the 64-bit block in a random direction."""
    f = Ffn(140, 72, 56, "fp16", "gelu_tanh", True, "fp32", seed=8)
    f.forward()
    f.backward()
    dy = f.dy.double()

    def loss(x, gu, d):
        g, u = x @ gu[:56].t(), x @ gu[56:].t()
        return ((R.ACTS["gelu_tanh"](g) * u) @ d.t() * dy).sum()

    at = [t.double() for t in (f.x, f.gate_up, f.down)]
    want = f.want(True)
    for i, (name, got) in enumerate((("dx", f.dx), ("dgate_up", f.dgate_up), ("ddown", f.ddown))):
        way = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=gen(i)) * 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + way, at[i] - way
        diff = (loss(*up) - loss(*down)) / 2
        # what roundings may do along the way, and the differences' third-order term
        assert abs((got.double() * way).sum() - diff) <= (want[name][1] * way.abs()).sum() + 1e-6 * (want[name][0].abs() * way.abs()).sum()


def test_ffn_repeats_bitwise_and_on_another_stream():
    f = Ffn(300, 264, 520, "bf16", "silu", True, seed=9)
    f.forward()
    f.backward()
    torch.cuda.synchronize()
    first = [t.clone() for t in (f.y, f.dx, f.dgate_up, f.ddown)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in (f.y, f.dx, f.dgate_up, f.ddown):
            t.zero_()
        f.forward()
        f.backward()
    side.synchronize()
    for a, b in zip(first, (f.y, f.dx, f.dgate_up, f.ddown)):
        assert torch.equal(a, b)


def test_ffn_no_tokens():
    f = Ffn(0, 64, 48, "bf16", "silu", True, seed=1)
    f.plan.forward(0, 0, 0, 0, 0, stream())
    f.plan.backward(0, 0, 0, 0, 0, 0, f.dgu0.data_ptr(), f.dd0.data_ptr(), 1, stream())
    assert (f.dgate_up == 7.0).all() and (f.ddown == 7.0).all()
    f.plan.backward(0, 0, 0, 0, 0, 0, f.dgu0.data_ptr(), f.dd0.data_ptr(), 0, stream())
    assert (f.dgate_up == 0.0).all() and (f.ddown == 0.0).all()


def test_ffn_large_gates():
    """Gates far in both tails: act' of a large gate whose cube overflows is 1 or 0, not NaN."""
    for act in ACT:
        f = Ffn(130, 64, 64, "bf16", act, True, "fp32", seed=2)
        f.gate_up[:64] *= 1e15 if act == "gelu_tanh" else 1e3
        f.down *= 2.0 ** -60 if act == "gelu_tanh" else 1.0
        f.forward()
        f.backward()
        f.plan.check()
        for t in (f.y, f.dx, f.dgate_up, f.ddown):
            assert torch.isfinite(t.float()).all(), act


# ---------------------------------------------------------------- cross entropy
class Ce:
    def __init__(self, T, H, V, dtype, train, smoothing=0.0, ignore=-100, grad="same", lds=(0, 0), keep=-1, piece=0, seed=0, spread=2.0):
        dt, code = DT[dtype]
        g = gen(seed)
        self.x0, self.x = strided(T, H, dt, g, lds[0])
        self.w0, self.w = strided(V, H, dt, g, lds[1], spread * H ** -0.5)
        self.target = torch.randint(0, V, (T,), device="cuda", generator=g)
        self.loss, self.lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
        self.dloss = (0.5 + torch.rand(T, device="cuda", generator=g)) * (1024.0 if dtype == "fp16" else 1.0) / max(1, T)
        gt, gcode = (torch.float32, E.FP32) if grad == "fp32" else (dt, code)
        self.dx0, self.dx = strided(T, H, dt, None, lds[0], fill=7.0)
        self.dw0, self.dw = strided(V, H, gt, None, lds[1], fill=7.0)
        self.smoothing, self.ignore, self.kept = smoothing, ignore, keep != 0
        self.plan = E.CePlan(E.CeDesc(T, H, V, code, int(train), gcode, smoothing, ignore, lds[0], lds[1], keep, piece))
        self.saved = torch.full((self.plan.saved_bytes() + 256,), 255, device="cuda", dtype=torch.uint8)

    def forward(self, saved=True):
        self.plan.forward(self.x0.data_ptr(), self.w0.data_ptr(), self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(),
                          self.saved.data_ptr() if saved else 0, stream())

    def backward(self, accumulate=0, dx=True, dw=True):
        self.plan.backward(self.x0.data_ptr(), self.w0.data_ptr(), self.target.data_ptr(), self.lse.data_ptr(), self.dloss.data_ptr(),
                           self.saved.data_ptr(), self.dx0.data_ptr() if dx else 0, self.dw0.data_ptr() if dw else 0, accumulate, stream())

    def want(self, train):
        return R.ce(self.x, self.w, self.target, self.smoothing, self.ignore, self.dloss if train else None, self.kept)

    def check(self, want):
        self.plan.check()
        R.check(self.loss, want["loss"], "loss")
        R.check(self.lse, want["lse"], "lse")
        if "dx" in want:
            R.check(self.dx, want["dx"], "dx")
            R.check(self.dw, R.rounded(want["dw"], self.dw.dtype), "dw")
            assert (self.dx0[self.dx.shape[0]:] == 7.0).all() and (self.dw0[self.dw.shape[0]:] == 7.0).all()
        assert (self.saved[self.plan.saved_bytes():] == 255).all()


CE_SIZES = [(1, 64, 64), (1, 8, 1), (3, 1, 5), (140, 1, 2), (20, 2120, 900), (100, 1096, 70), (2, 72, 7), (31, 136, 1000), (33, 264, 5001), (128, 520, 20011), (129, 264, 1003), (300, 72, 513), (513, 1032, 4099)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,H,V", CE_SIZES)
def test_ce_forward(T, H, V, dtype):
    for smoothing in (0.0, 0.1):
        c = Ce(T, H, V, dtype, False, smoothing, seed=V)
        c.target[::3] = -100
        c.forward(saved=False)
        c.check(c.want(False))


@pytest.mark.parametrize("T,H,V,dtype,smoothing,grad,keep,piece", [
    (1, 64, 64, "bf16", 0.0, "same", -1, 0), (2, 72, 7, "fp16", 0.1, "fp32", -1, 0), (100, 136, 3001, "bf16", 0.1, "fp32", -1, 0),
    (100, 136, 3001, "bf16", 0.0, "same", 0, 0), (129, 264, 1003, "fp16", 0.0, "same", -1, 0), (300, 72, 2050, "bf16", 0.0, "fp32", 0, 256),
    (300, 72, 2050, "fp16", 0.1, "fp32", 700000, 256), (513, 520, 4099, "bf16", 0.0, "same", 1800000, 1000), (64, 136, 3001, "bf16", 0.0, "same", 250000, 0),
    (1, 64, 2000, "fp16", 0.0, "fp32", 0, 512)])
def test_ce_training(T, H, V, dtype, smoothing, grad, keep, piece):
    c = Ce(T, H, V, dtype, True, smoothing, grad=grad, keep=keep, piece=piece, seed=T + V)
    if keep > 0:
        assert 0 < c.plan.saved_bytes() <= keep   # a part of the vocabulary is kept, the rest recomputed
    c.target[1::4] = -100
    c.forward()
    c.backward()
    c.check(c.want(True))


@pytest.mark.parametrize("T,lds", [(5, (65, 67)), (140, (65, 67)), (140, (72, 67)), (140, (80, 96))])
def test_ce_strides(T, lds):
    c = Ce(T, 65, 333, "bf16", True, lds=lds, seed=4)
    c.forward()
    c.backward()
    c.check(c.want(True))
    assert (c.dx0[:, 65:] == 7.0).all() and (c.dw0[:, 65:] == 7.0).all()


def test_ce_targets():
    """Ignored targets, targets outside the vocabulary, one target many times, the first and the last column."""
    c = Ce(140, 72, 515, "bf16", True, ignore=3, seed=6)
    c.target[:20] = 3
    c.target[20:25] = torch.tensor([-1, 515, 1 << 40, -(1 << 40), -100], device="cuda")
    c.target[25:60] = 514
    c.target[60:90] = 0
    c.dloss[:5] = float("nan")   # of ignored rows: not read into anything
    c.forward()
    c.backward()
    want = R.ce(c.x, c.w, c.target, 0.0, 3, torch.where(torch.isnan(c.dloss), torch.zeros_like(c.dloss), c.dloss), True)
    c.check(want)
    assert (c.loss[:25] == 0).all() and (c.dx[:25] == 0).all()
    c.target.fill_(-100)         # nothing to learn
    c.forward()
    c.backward()
    c.plan.check()
    for t in (c.loss, c.dx, c.dw):
        assert (t == 0).all()


@pytest.mark.parametrize("T", [100, 140])
def test_ce_large_logits(T):
    """Logits of some thousands, of both signs: only differences from the largest are exponentiated."""
    c = Ce(T, 64, 1000, "bf16", True, spread=400.0, grad="fp32", seed=7)
    c.forward()
    c.backward()
    c.plan.check()
    want = c.want(False)
    R.check(c.loss, want["loss"])
    R.check(c.lse, want["lse"])
    assert torch.isfinite(c.dx.float()).all() and torch.isfinite(c.dw).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1.0, 1e20])
def test_ce_gradient_scale(scale):
    """dloss of any size: the gradients scale with it (fp32 and bf16 results), zeros among it."""
    c = Ce(140, 72, 515, "bf16", True, grad="fp32", seed=10)
    c.forward()
    c.backward()
    small, small_x = c.dw.clone(), c.dx.float()
    two = 2.0 ** round(torch.log2(torch.tensor(scale)).item())
    c.dloss *= two
    c.forward()
    c.backward()
    assert torch.equal(c.dw, small * two) and torch.equal(c.dx.float(), small_x * two)   # powers of two round nothing
    c.dloss[:] = 0
    c.forward()
    c.backward()
    assert (c.dw == 0).all() and (c.dx == 0).all()


def test_ce_accumulates_and_leaves_out():
    for keep in (-1, 0):
        c = Ce(140, 72, 515, "bf16", True, grad="fp32", keep=keep, piece=256, seed=11)
        c.forward()
        c.backward()
        dx, dw = c.dx.clone(), c.dw.clone()
        c.forward()
        c.backward(accumulate=1)
        assert torch.equal(c.dw, 2 * dw) and torch.equal(c.dx, dx)
        c.dx.fill_(5.0)
        c.dw.fill_(5.0)
        c.forward()
        c.backward(dx=False)
        assert (c.dx == 5.0).all() and torch.equal(c.dw, dw)
        c.dw.fill_(5.0)
        c.forward()
        c.backward(dw=False)
        assert (c.dw == 5.0).all() and torch.equal(c.dx, dx)


def test_ce_gradient_against_differences():
    c = Ce(140, 72, 300, "fp16", True, 0.1, grad="fp32", seed=12)
    c.forward()
    c.backward()
    want = c.want(True)

    def loss(x, w):
        l = x @ w.t()
        hit = l.gather(1, c.target[:, None])[:, 0]
        return ((torch.logsumexp(l, 1) - 0.9 * hit - 0.1 * l.mean(1)) * c.dloss.double()).sum()

    at = [c.x.double(), c.w.double()]
    for i, (name, got) in enumerate((("dx", c.dx), ("dw", c.dw))):
        way = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=gen(i)) * 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + way, at[i] - way
        diff = (loss(*up) - loss(*down)) / 2
        assert abs((got.double() * way).sum() - diff) <= (want[name][1] * way.abs()).sum() + 1e-6 * (want[name][0].abs() * way.abs()).sum()


def test_ce_repeats_bitwise():
    for keep in (-1, 0):
        c = Ce(300, 264, 2051, "bf16", True, keep=keep, piece=512, seed=13)
        runs = []
        for _ in range(2):
            c.forward()
            c.backward()
            torch.cuda.synchronize()
            runs.append([t.clone() for t in (c.loss, c.lse, c.dx, c.dw)])
            for t in (c.loss, c.lse, c.dx, c.dw):
                t.zero_()
        assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_ce_no_tokens():
    c = Ce(0, 64, 48, "bf16", True, seed=1)
    c.plan.forward(0, 0, 0, 0, 0, 0, stream())
    c.plan.backward(0, 0, 0, 0, 0, 0, 0, c.dw0.data_ptr(), 0, stream())
    assert (c.dw == 0).all()


# ---------------------------------------------------------------- 8-bit integers
def codes_of(rows, K, g):
    ld = (K + 15) // 16 * 16 + 16 * (K % 2)
    c = torch.randint(-128, 128, (rows, ld), device="cuda", dtype=torch.int8, generator=g)
    s = torch.rand(rows, device="cuda", generator=g) + 0.5
    return c, s, E.I8(rows, K, ld, c.data_ptr(), s.data_ptr())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,K,ldx", [(1, 1, 1), (1, 8192, 8192), (3, 37, 40), (5, 4100, 4100), (200, 1000, 1001), (7, 129, 136), (2, 0, 1)])
def test_i8_quantize(rows, K, ldx, dtype):
    code = {torch.bfloat16: E.BF16, torch.float16: E.FP16, torch.float32: E.FP32}[dtype]
    x0, x = strided(rows, K, dtype, gen(K), ldx)
    if rows > 2 and K:
        x[1] = 0                                          # a row of zeros
        x[2, :] = torch.arange(K, device="cuda") % 255 - 127.0   # ties and exact codes
    ld = (K + 15) // 16 * 16 + 16
    codes, scales = torch.full((rows, ld), 99, device="cuda", dtype=torch.int8), torch.full((rows,), -1.0, device="cuda")
    E.I8(rows, K, ld, codes.data_ptr(), scales.data_ptr()).quantize(x0.data_ptr(), ldx, code, stream())
    want, ws = R.quantized(x)
    assert torch.equal(scales.cpu(), ws) and torch.equal(codes[:, :K].cpu(), want)
    assert (codes[:, K:] == 99).all()


def test_i8_quantize_ties_and_tiny():
    """Quotients on and next to ties, scales among the subnormal numbers."""
    g = gen(1)
    scale = torch.rand(64, 1, device="cuda", generator=g) + 0.5
    half = torch.randint(-253, 254, (64, 512), device="cuda", generator=g) / 2.0
    x = half * scale
    x = torch.where(torch.rand(64, 512, device="cuda", generator=g) < 0.5, torch.nextafter(x, torch.zeros_like(x)), x)
    x[:, 0] = 127 * scale[:, 0]
    x[40:50] *= 2.0 ** -130
    x[50:60] *= 2.0 ** -142
    x[60:] *= 2.0 ** -148
    codes, scales = torch.empty(64, 512, device="cuda", dtype=torch.int8), torch.empty(64, device="cuda")
    E.I8(64, 512, 512, codes.data_ptr(), scales.data_ptr()).quantize(x.data_ptr(), 512, E.FP32, stream())
    want, ws = R.quantized(x)
    assert torch.equal(scales.cpu(), ws) and torch.equal(codes.cpu(), want)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 300, 64), (3, 5001, 33), (16, 257, 1040), (37, 640, 4100), (128, 2403, 129), (129, 257, 40),
                                   (2, 64, 8192), (50, 272, 3100), (100, 1030, 4128), (300, 520, 1000), (300, 523, 1000), (257, 132, 64), (1000, 130, 272), (64, 35, 64), (65, 37, 272)])
def test_i8_gemm(M, N, K, out):
    g = gen(M + N)
    (xc, xs, X), (wc, ws, W) = codes_of(M, K, g), codes_of(N, K, g)
    code = {torch.bfloat16: E.BF16, torch.float16: E.FP16, torch.float32: E.FP32}[out]
    sums = xc[:, :K].double() @ wc[:, :K].double().t()
    real = sums * xs.double()[:, None] * ws.double()[None]
    alpha = 2.0 ** -8 if out == torch.float16 else 1.0     # (results of some 10^5 are beyond fp16)
    alpha = alpha * 2.0 ** -6 if out == torch.float16 and K > 1000 else alpha
    for ldy in (N, N + 5, (N + 31) // 32 * 32 + 32):
        y0, y = strided(M, N, out, None, ldy, fill=7.0)
        W.gemm(X, y0.data_ptr(), ldy, code, alpha, 0.0, stream())
        assert E.exo_fused_check() == E.OK
        # the sum's conversion and three products are rounded to 24 bits, the result to its type
        bound = 4 * 2.0 ** -24 * (alpha * real).abs()
        R.check(y, R.rounded((alpha * real, bound), out))
        assert (y0[:, N:] == 7.0).all() and (y0[M:] == 7.0).all()
    _, y1 = strided(M, N, out, g, 0)
    before = y1.double()
    W.gemm(X, y1.data_ptr(), N, code, alpha, 0.5, stream())
    want = alpha * real + 0.5 * before
    R.check(y1, R.rounded((want, 6 * 2.0 ** -24 * ((alpha * real).abs() + before.abs())), out))


def test_i8_extremes():
    """Sums at both ends of 32 bits, and rows that are far from the start of a large matrix."""
    K = 131071
    ld = 131072
    x = torch.full((2, ld), -128, device="cuda", dtype=torch.int8)
    w = torch.full((17, ld), -128, device="cuda", dtype=torch.int8)
    w[3] = 127
    s = torch.ones(17, device="cuda")
    y = torch.empty(2, 17, device="cuda")
    E.I8(17, K, ld, w.data_ptr(), s.data_ptr()).gemm(E.I8(2, K, ld, x.data_ptr(), s.data_ptr()), y.data_ptr(), 17, E.FP32, stream=stream())
    want = torch.full((2, 17), float(K * 16384), device="cuda")
    want[:, 3] = float(-K * 128 * 127)
    assert torch.equal(y, want)
    rows = (1 << 32) // 16384 + 100      # codes beyond 2^32 bytes
    w = torch.ones(rows, 16384, device="cuda", dtype=torch.int8)
    w[-1] = 2
    s = torch.ones(rows, device="cuda")
    y = torch.empty(2, rows, device="cuda")
    E.I8(rows, 16384, 16384, w.data_ptr(), s.data_ptr()).gemm(E.I8(2, 16384, ld, x.data_ptr(), s.data_ptr()), y.data_ptr(), rows, E.FP32, stream=stream())
    assert (y[:, :-1] == -128 * 16384).all() and (y[:, -1] == -256 * 16384).all()


def test_i8_without_products():
    g = gen(3)
    (_, _, X), (_, _, W) = codes_of(5, 64, g), codes_of(33, 64, g)
    for dt, code in ((torch.float32, E.FP32), (torch.bfloat16, E.BF16), (torch.float16, E.FP16)):
        y = torch.ones(5, 33, device="cuda", dtype=dt)
        W.gemm(X, y.data_ptr(), 33, code, 0.0, 0.5, stream())
        assert (y == 0.5).all()
        y.fill_(float("nan"))
        E.I8(33, 0, 64, W.struct.codes, W.struct.scales).gemm(E.I8(5, 0, 64, 0, 0), y.data_ptr(), 33, code, 1.0, 0.0, stream())
        assert (y == 0).all()


# ---------------------------------------------------------------- together, captured, and waits that run out
def training_step(f, c):
    """A block and the head over its output, forward and backward."""
    f.forward()
    c.plan.forward(f.y0.data_ptr(), c.w0.data_ptr(), c.target.data_ptr(), c.loss.data_ptr(), c.lse.data_ptr(), c.saved.data_ptr(), stream())
    c.plan.backward(f.y0.data_ptr(), c.w0.data_ptr(), c.target.data_ptr(), c.lse.data_ptr(), c.dloss.data_ptr(), c.saved.data_ptr(), f.dy0.data_ptr(),
                    c.dw0.data_ptr(), 0, stream())
    f.backward()


@pytest.mark.parametrize("T,F,lds,keep", [(200, 264, (0, 0, 0, 0), 300000), (200, 261, (0, 0, 0, 0), 300000), (40, 261, (0, 0, 0, 0), -1),
                                          (40, 264, (0, 0, 139, 0), 0)])
def test_a_training_step_and_its_graph(T, F, lds, keep):
    f = Ffn(T, 136, F, "bf16", "silu", True, lds=lds, seed=21)
    c = Ce(T, 136, 1003, "bf16", True, keep=keep, piece=256, seed=22)
    training_step(f, c)
    torch.cuda.synchronize()
    outs = lambda: (f.y, f.dy, f.dx, f.dgate_up, f.ddown, c.loss, c.dw)  # noqa: E731
    first = [t.clone() for t in outs()]
    # each operator on what the one before it left
    want = R.ce(f.y, c.w, c.target, dloss=c.dloss, kept=keep != 0)
    R.check(c.loss, want["loss"])
    R.check(f.dy, want["dx"])
    f.check_backward(f.want(True))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            training_step(f, c)
    for _ in range(2):
        for t in outs():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs()))
    f.x.copy_(torch.randn(f.x.shape, device="cuda", generator=gen(99)))   # other inputs in the same places
    graph.replay()
    torch.cuda.synchronize()
    f.check_backward(f.want(True))


def test_first_calls_may_be_captured():
    """In a process of its own: nothing has been launched before the capture, so kernels are loaded under it."""
    import os
    import subprocess
    import sys
    code = """
import torch, test_fused_gpu as T
from paper_2609_16389_b200 import fused as E
f, c = T.Ffn(70, 136, 261, "bf16", "silu", True, seed=21), T.Ce(70, 136, 1003, "bf16", True, keep=100000, piece=256, seed=22)
(_, _, W), x = T.codes_of(136, 136, T.gen(1)), torch.randn(70, 136, device="cuda").bfloat16()
codes, scales, y = torch.empty(70, 144, device="cuda", dtype=torch.int8), torch.empty(70, device="cuda"), torch.empty(70, 136, device="cuda")
X = E.I8(70, 136, 144, codes.data_ptr(), scales.data_ptr())
torch.cuda.synchronize()
graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
    T.training_step(f, c)
    X.quantize(x.data_ptr(), 136, E.BF16, T.stream())
    W.gemm(X, y.data_ptr(), 136, E.FP32, stream=T.stream())
graph.replay()
torch.cuda.synchronize()
f.check_backward(f.want(True))
assert torch.isfinite(y).all() and y.abs().max() > 0
"""
    tests = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join((os.path.dirname(tests), tests)))
    assert subprocess.run([sys.executable, "-c", code], env=env, timeout=300).returncode == 0


def test_plans_side_by_side():
    """Two plans at once on two streams: they share nothing."""
    pairs = [(Ffn(150, 136, 264, "bf16", "silu", True, seed=s), Ce(150, 136, 515, "bf16", True, seed=s + 1), torch.cuda.Stream()) for s in (30, 40)]
    torch.cuda.synchronize()
    for _ in range(3):
        for f, c, side in pairs:
            with torch.cuda.stream(side):
                training_step(f, c)
    torch.cuda.synchronize()
    for f, c, _ in pairs:
        f.check_backward(f.want(True))


def test_example():
    """It runs, and its gradients are those of automatic differentiation up to five roundings to bf16 (2^-8 each at most)."""
    from examples import train_step
    step = train_step.Step(140, 136, 200, 515)
    loss, grads = step.by_autograd()
    got = step.forward()
    step.backward()
    step.block.check()
    step.loss_head.check()
    assert abs(got.item() - loss.item()) <= 2.0 ** -8 * loss.item()
    for a, b in zip((step.dx, step.d_gate_up, step.d_down, step.d_head), grads):
        assert train_step.off(a, b) <= 5 * 2.0 ** -8
    step.update(0.1)
    logits, want = step.scores_in_8_bits()
    assert logits.shape == want.shape and torch.isfinite(logits).all()


def test_refusals_on_plans():
    f = Ffn(20, 64, 48, "bf16", "silu", True, lds=(0, 0, 0, 51), seed=1)
    x, gu, d, y, s, dy = (t.data_ptr() for t in (f.x0, f.gu0, f.d0, f.y0, f.saved, f.dy0))
    dx, dgu, dd = f.dx0.data_ptr(), f.dgu0.data_ptr(), f.dd0.data_ptr()
    h = f.plan.handle
    for args, status in (((0, gu, d, y, s), 1), ((x, 0, d, y, s), 1), ((x, gu, 0, y, s), 1), ((x, gu, d, 0, s), 1), ((x + 2, gu, d, y, s), 4),
                         ((x, gu + 8, d, y, s), 4), ((x, gu, d + 1, y, s), 4), ((x, gu, d, y + 4, s), 4), ((x, gu, d, y, s + 16), 4)):
        assert E.exo_ffn_forward(h, *args, stream()) == status
    for args, status in (((x, gu, 0, s, dy, dx, dgu, dd), 1), ((x, gu, d, 0, dy, dx, dgu, dd), 1), ((x, gu, d, s, 0, dx, dgu, dd), 1),
                         ((0, gu, d, s, dy, dx, dgu, dd), 1), ((x, 0, d, s, dy, dx, dgu, dd), 1), ((x, gu, d, s + 16, dy, dx, dgu, dd), 4),
                         ((x, gu, d, s, dy + 2, dx, dgu, dd), 4), ((x, gu, d, s, dy, dx + 8, dgu, dd), 4), ((x, gu, d, s, dy, dx, dgu + 4, dd), 4),
                         ((x, gu, d, s, dy, dx, dgu, dd + 1), 4)):
        assert E.exo_ffn_backward(h, *args, 0, stream()) == status
    assert E.exo_ffn_backward(h, 0, 0, 0, 0, 0, 0, 0, 0, 0, stream()) == 0           # nothing wanted
    c = Ce(20, 64, 48, "bf16", True, lds=(0, 67), seed=1)
    x, w, t, lo, ls, s, dl = (v.data_ptr() for v in (c.x0, c.w0, c.target, c.loss, c.lse, c.saved, c.dloss))
    dx, dw = c.dx0.data_ptr(), c.dw0.data_ptr()
    h = c.plan.handle
    for args, status in (((0, w, t, lo, ls, s), 1), ((x, 0, t, lo, ls, s), 1), ((x, w, 0, lo, ls, s), 1), ((x + 2, w, t, lo, ls, s), 4),
                         ((x, w + 1, t, lo, ls, s), 4), ((x, w, t + 4, lo, ls, s), 4), ((x, w, t, lo + 2, ls, s), 4), ((x, w, t, lo, ls + 2, s), 4),
                         ((x, w, t, lo, ls, s + 4), 4)):
        assert E.exo_ce_forward(h, *args, stream()) == status
    for args, status in (((0, w, t, ls, dl, s, dx, dw), 1), ((x, 0, t, ls, dl, s, dx, dw), 1), ((x, w, 0, ls, dl, s, dx, dw), 1),
                         ((x, w, t, 0, dl, s, dx, dw), 1), ((x, w, t, ls, 0, s, dx, dw), 1), ((x, w, t, ls, dl, 0, dx, dw), 1),
                         ((x, w, t, ls, dl, s + 8, dx, dw), 4), ((x, w, t, ls, dl, s, dx + 2, dw), 4), ((x, w, t, ls, dl, s, dx, dw + 1), 4)):
        assert E.exo_ce_backward(h, *args, 0, stream()) == status
    for kind, plan in (("ffn", Ffn(20, 64, 48, "bf16", "silu", False).plan), ("ce", Ce(20, 64, 48, "bf16", False).plan)):
        assert plan.saved_bytes() == 0
    g = Ffn(20, 64, 48, "bf16", "silu", False)
    p = g.x0.data_ptr()
    assert E.exo_ffn_forward(g.plan.handle, p, p, p, p, p, stream()) == 2            # a plan that does not train keeps nothing
    assert E.exo_ffn_backward(g.plan.handle, p, p, p, p, p, p, p, p, 0, stream()) == 2
    assert E.exo_fused_check() == 0


@pytest.mark.parametrize("T", [4, 200])
def test_a_wait_that_runs_out_is_reported(T):
    f = Ffn(T, 264, 136, "bf16", "silu", False, seed=1)
    f.forward(saved=False)
    torch.cuda.synchronize()
    good = f.y.clone()
    assert E.exo_fused_debug_set(20, 1) == E.OK
    f.forward(saved=False)
    assert E.exo_fused_check() == 7
    f.plan.close()
    g = Ffn(T, 264, 136, "bf16", "silu", False, seed=1)
    g.forward(saved=False)
    g.plan.check()
    assert torch.equal(g.y, good)


def test_ce_keeps_rare_columns_in_fp16():
    """Peaked rows: most columns' probabilities lie far below fp16's smallest part of the row's largest, and the kept exponentials still hold them."""
    c = Ce(140, 72, 1000, "fp16", True, grad="fp32", seed=15, spread=6.0)
    c.forward()
    c.backward()
    bare = R.ce(c.x, c.w, c.target, dloss=c.dloss, kept=False)
    # what keeping may add: half a step of the exponential, relative, and half of fp16's smallest step where the row's largest is 2^15
    l = c.x.double() @ c.w.double().t()
    p = torch.softmax(l, 1)
    kept = c.dloss.double()[:, None] * (p * 2.0 ** -11 + 2.0 ** -40 * p.amax(1, keepdim=True)) * (1 + 2.0 ** -10)
    assert (p < 1e-7 * p.amax(1, keepdim=True)).double().mean() > 0.3
    c.check({"loss": bare["loss"], "lse": bare["lse"], "dx": (bare["dx"][0], bare["dx"][1] + (1 + 2.0 ** -10) * (kept @ c.w.double().abs())),
             "dw": (bare["dw"][0], bare["dw"][1] + kept.t() @ c.x.double().abs())})


@pytest.mark.parametrize("T", [4, 200])
def test_a_wait_that_runs_out_is_its_own_plans(T):
    """Of two plans, the one whose wait ran out reports that, whoever is asked first; the other's results are right and it reports nothing."""
    for first in (0, 1):
        pair = [Ffn(T, 264, 136, "bf16", "silu", True, seed=s) for s in (1, 2)]
        heads = [Ce(T, 264, 515, "bf16", True, seed=s) for s in (1, 2)]
        for broken, well, want in (pair + [lambda o: R.check(o.y, o.want(False)["y"])], heads + [lambda o: R.check(o.lse, o.want(False)["lse"])]):
            well.forward()
            torch.cuda.synchronize()
            assert E.exo_fused_debug_set(20, 1) == E.OK
            broken.forward()
            well.forward()
            for o in ((broken, well), (well, broken))[first]:
                if o is broken:
                    with pytest.raises(E.ExoGemmError) as e:
                        o.plan.check()
                    assert e.value.status == 7
                else:
                    o.plan.check()
                    want(o)
            broken.forward()          # it has been asked: the next call is as good as any
            broken.plan.check()
            want(broken)
        assert E.exo_fused_check() == 7 and E.exo_fused_check() == E.OK   # of the device, since it was asked last


def test_a_wait_of_an_8_bit_product_is_no_plans():
    f = Ffn(40, 264, 136, "bf16", "silu", False, seed=1)
    (_, _, X), (_, _, W) = codes_of(5, 640, gen(1)), codes_of(33, 640, gen(2))
    y = torch.zeros(5, 33, device="cuda")
    assert E.exo_fused_debug_set(20, 1) == E.OK
    W.gemm(X, y.data_ptr(), 33, E.FP32, stream=stream())
    f.forward(saved=False)
    f.check_forward(f.want(False))
    assert E.exo_fused_check() == 7 and E.exo_fused_check() == E.OK


@pytest.mark.parametrize("T,keep", [(40, -1), (200, 300000)])
def test_ce_second_backward_is_not_taken_for_a_gradient(T, keep):
    """The kept exponentials serve one backward call: a second one, or one without its forward call, gives NaN and no numbers."""
    c = Ce(T, 72, 1003, "bf16", True, keep=keep, piece=256, seed=16)
    assert 0 < c.plan.saved_bytes() and (keep < 0 or c.plan.saved_bytes() <= keep)
    c.forward(saved=False)
    c.backward()                       # nothing has been left in `saved`
    assert c.dx.isnan().all() and c.dw.isnan().all()
    c.forward()
    c.backward()
    c.check(c.want(True))
    dx, dw = c.dx.clone(), c.dw.clone()
    c.backward()
    assert c.dx.isnan().all() and c.dw.isnan().all()
    c.forward()
    c.backward()
    assert torch.equal(c.dx, dx) and torch.equal(c.dw, dw)


# ---------------------------------------------------------------- values where functions saturate
@pytest.mark.parametrize("T", [20, 130])
@pytest.mark.parametrize("act", ACT)
def test_ffn_values_in_the_gates_tails(act, T):
    """Gates far in both tails, exact since a token has a single value, 1: there act is g or 0 and its slope 1 or 0, also where exponentials, and
    the cube of a gate, overflow."""
    H, F = 64, 72
    f = Ffn(T, H, F, "bf16", act, True, "fp32", seed=2)
    at = torch.arange(T, device="cuda")
    f.x.zero_()
    f.x[at, at % H] = 1
    g0 = gen(3)
    f.gate_up[:F] = torch.sign(torch.randn(F, H, device="cuda", generator=g0)) * 2.0 ** torch.randint(7, 10, (F, H), device="cuda", generator=g0)
    if act == "gelu_tanh":
        f.gate_up[:F] *= 2.0 ** 50
    f.forward()
    f.backward()
    f.plan.check()
    dt = f.x.dtype
    g, u = (w[:, at % H].t().double() for w in (f.gate_up[:F], f.gate_up[F:]))
    up = (g > 0).double()
    # a sigmoid next to 1 may be a step of fp32 off, which its factor g multiplies in the slope
    a, slope = (g * up, R.FUNCTION * g * up), (up, R.FUNCTION * (1 + g.abs().clamp(max=1024.0) * up))
    X, Wg, Wu, Wd, dY, U = R.exactly(f.x), R.exactly(f.gate_up[:F]), R.exactly(f.gate_up[F:]), R.exactly(f.down), R.exactly(f.dy), R.exactly(u)
    h = R.rounded(R.product(a, U), dt)
    R.check(f.y, R.rounded(R.matmul(h, R.turned(Wd)), dt), "y")
    dh = R.matmul(dY, Wd)
    dg, du = R.rounded(R.product(R.product(dh, U), slope), dt), R.rounded(R.product(dh, a), dt)
    dx = R.plus(R.matmul(dg, Wg), R.matmul(du, Wu))
    m = (dg[0].abs() + dg[1]) @ Wg[0].abs() + (du[0].abs() + du[1]) @ Wu[0].abs()
    R.check(f.dx, R.rounded((dx[0], dx[1] + 2 * F * 2.0 ** -23 * m), dt), "dx")   # one sum of 2 F products
    dgu = [R.matmul(R.turned(t), X) for t in (dg, du)]
    R.check(f.dgate_up, (torch.cat([t[0] for t in dgu]), torch.cat([t[1] for t in dgu])), "dgate_up")
    R.check(f.ddown, R.matmul(R.turned(dY), h), "ddown")
    assert (f.dgate_up[:F][(f.gate_up[:F] < 0) & (torch.arange(H, device="cuda") < T)] == 0).all()   # nothing flows through a closed gate


@pytest.mark.parametrize("T,keep", [(100, -1), (140, -1), (140, 0)])
def test_ce_gradients_of_large_logits(T, keep):
    """Logits of some thousands: a row's gradient is at its target and its largest column, and nowhere where these are one."""
    c = Ce(T, 64, 1000, "bf16", True, spread=400.0, grad="fp32", keep=keep, piece=256, seed=7)
    at = torch.arange(T, device="cuda")
    c.x.zero_()
    c.x[at, at % 64] = 32
    l = c.x.double() @ c.w.double().t()
    c.target[::2] = l.argmax(1)[::2]
    c.forward()
    c.backward()
    want = c.want(True)
    # an exponential below fp32's smallest normal number, 2^-126, may be lost: that much of every column, times the row's |dloss|
    lost = (c.dloss.double()[:, None] * 2.0 ** -126).expand(T, 1000)
    want["dx"] = want["dx"][0], want["dx"][1] + lost @ c.w.double().abs()
    want["dw"] = want["dw"][0], want["dw"][1] + lost.t() @ c.x.double().abs()
    c.check(want)
    d = torch.softmax(l, 1) - torch.nn.functional.one_hot(c.target, 1000)
    assert l.abs().max() > 4000 and (d.abs().sum(1) > 1.9).any() and (d.abs().sum(1) < 1e-6).any()


# ---------------------------------------------------------------- several tiles to a pair of CTAs
# On 148 SMs (74 pairs) these take tiles of 64 to 256 columns, up to thirteen to a pair: both accumulators and their hand-over, rings that run on
# from tile to tile, bands of several tile columns, results whose buffers are used again.
@pytest.mark.parametrize("T,H,F,dtype,act,grad", [
    (600, 264, 3104, "bf16", "silu", "same"),        # 147 tiles of 128 gated columns
    (900, 136, 9541, "fp16", "gelu", "fp32"),        # 400 of 192, rows of odd length; 152 of 256 in the backward pass
    (1100, 200, 11456, "bf16", "gelu_tanh", "fp32"),  # 450 of 256
    (1300, 136, 6254, "fp16", "silu", "same"),       # 294 of 128 in the backward pass
    (2600, 72, 774, "bf16", "silu", "fp32")])        # many rows, few columns
def test_ffn_many_tiles(T, H, F, dtype, act, grad):
    f = Ffn(T, H, F, dtype, act, True, grad, seed=F)
    f.forward()
    f.backward()
    want = f.want(True)
    f.check_forward(want)
    f.check_backward(want)


@pytest.mark.parametrize("T,H,V,dtype,smoothing,keep,piece", [
    (600, 136, 6254, "bf16", 0.1, -1, 0),            # 147 tiles of 128
    (900, 72, 9541, "fp16", 0.0, -1, 0),             # 200 of 192
    (1100, 136, 40003, "bf16", 0.0, -1, 0),          # 785 of 256
    (1100, 136, 40003, "fp16", 0.1, 0, 20000),       # pieces of several tiles to a pair
    (900, 264, 23000, "bf16", 0.0, 12000000, 9541)])  # a part kept, the rest recomputed
def test_ce_many_tiles(T, H, V, dtype, smoothing, keep, piece):
    c = Ce(T, H, V, dtype, True, smoothing, grad="fp32", keep=keep, piece=piece, seed=V)
    c.target[::5] = -100
    c.forward()
    c.backward()
    c.check(c.want(True))


@pytest.mark.parametrize("M,N,K", [(600, 6254, 200), (900, 9544, 130), (1100, 11460, 1040), (2600, 1030, 272)])
def test_i8_many_tiles(M, N, K):
    g = gen(N)
    (xc, xs, X), (wc, ws, W) = codes_of(M, K, g), codes_of(N, K, g)
    real = (xc[:, :K].double() @ wc[:, :K].double().t()) * xs.double()[:, None] * ws.double()[None]
    bound = 4 * 2.0 ** -24 * real.abs()   # the sum's conversion and three products
    for out, code in ((torch.bfloat16, E.BF16), (torch.float32, E.FP32)):
        for ldy in (N, (N + 31) // 32 * 32 + 32):     # rows that start anywhere, and on 16 bytes
            y0, y = strided(M, N, out, None, ldy, fill=7.0)
            W.gemm(X, y0.data_ptr(), ldy, code, 1.0, 0.0, stream())
            R.check(y, R.rounded((real, bound), out))
            assert (y0[:, N:] == 7.0).all() and (y0[M:] == 7.0).all()
            W.gemm(X, y0.data_ptr(), ldy, code, 1.0, 0.5, stream())
            twice = 1.5 * real, 6 * 2.0 ** -24 * 1.5 * real.abs() + (0.5 * R.half_step(out) * 1.01 * real.abs())   # beta times the rounded result
            R.check(y, R.rounded(twice, out))
    assert E.exo_fused_check() == E.OK
