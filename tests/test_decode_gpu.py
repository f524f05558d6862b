"""The few-token operators against their definitions in 64 bits.

Bounds, derived from the arithmetic and not from what the kernels give: a sum of n products that are exact in fp32,
accumulated in fp32 in some order with at most n / 8 + 32 roundings or truncations on the way of any term, is off by
at most (n / 8 + 32) * 2^-23 * sum |terms|; rounding to 16 bits adds u = 2^-8 (bf16) or 2^-11 (fp16) of the value, or
half the smallest subnormal number (2^-134, 2^-25).
"""
import numpy as np
import pytest

from paper_2609_16389_b200 import binding as B
from paper_2609_16389_b200 import decode as D

pytestmark = pytest.mark.gpu
U = {D.BF16: 2.0 ** -8, D.FP16: 2.0 ** -11, D.FP32: 2.0 ** -24}
TINY = {D.BF16: 2.0 ** -134, D.FP16: 2.0 ** -25, D.FP32: 0.0}


def torch():
    import torch as t
    return t


def tt(dtype):
    t = torch()
    return {D.BF16: t.bfloat16, D.FP16: t.float16, D.FP32: t.float32}[dtype]


def stream():
    return torch().cuda.current_stream().cuda_stream


def sum_bound(n):
    return (n / 8 + 32) * 2.0 ** -23


def groups(K, group):
    return D.padded_k(K) // group


class Matrix:
    """A 4-bit matrix on the device with its codes on the host; padding codes and all-padding groups hold junk."""

    def __init__(self, rows, K, group, dtype, zeros, seed, spread=0.02):
        t = torch()
        rng = np.random.default_rng(seed)
        self.rows, self.K, self.group, self.dtype = rows, K, group, dtype
        codes = rng.integers(0, 16, (rows, D.padded_k(K)), dtype=np.uint8)
        self.codes = t.from_numpy(D.pack_codes(codes)).cuda()
        G = groups(K, group)
        s = t.from_numpy(rng.uniform(0.2, 1.0, (rows, G)) * spread * rng.choice([-1, 1], (rows, G), p=[0.1, 0.9]))
        s[:, (K + group - 1) // group:] = float("nan")
        self.scales = s.to(tt(dtype)).cuda()
        self.zeros = t.from_numpy(rng.integers(0, 16, (rows, G), dtype=np.uint8)).cuda() if zeros else None
        z = self.zeros.cpu().numpy().astype(np.float64) if zeros else np.full((rows, G), 8.0)
        at = np.arange(K) // group
        self.values = (codes[:, :K].astype(np.float64) - z[:, at]) * self.scales.double().cpu().numpy()[:, at]

    def q4(self):
        return D.Q4(self.rows, self.K, self.group, self.dtype, self.codes.data_ptr(), self.scales.data_ptr(),
                    0 if self.zeros is None else self.zeros.data_ptr())


# ------------------------------------------------------------------ quantisation
QUANT = [(1, 1, 32, False), (3, 7, 32, True), (5, 127, 64, False), (2, 128, 128, True), (33, 260, 32, True),
         (4, 300, 128, False), (7, 4097, 64, True), (2, 9000, 128, False), (130, 512, 64, False)]


@pytest.mark.parametrize("rows,K,group,zeros", QUANT)
@pytest.mark.parametrize("dtype,src", [(D.BF16, D.BF16), (D.FP16, D.FP16), (D.BF16, D.FP32), (D.FP16, D.FP32), (D.FP16, D.BF16)])
def test_quantize_follows_its_formula_code_by_code(rows, K, group, zeros, dtype, src):
    t = torch()
    gen = t.Generator().manual_seed(rows * 1000 + K)
    ldw = K + 3
    w = t.full((rows, ldw), float("nan"))
    w[:, :K] = t.randn(rows, K, generator=gen) * t.exp(t.randn(rows, 1, generator=gen))
    if rows > 2:
        w[1, :K] = 0.0                       # a row of zeros: scale 0, code = zero
        w[2, :K] = w[2, :K].abs()            # one sign only
    w = w.to(tt(src))
    G, Kp = groups(K, group), D.padded_k(K)
    codes = t.full((rows + 1, Kp // 2), 0xa5, dtype=t.uint8, device="cuda")      # one row more than is written
    scales = t.full((rows + 1, G), 7.0, dtype=tt(dtype), device="cuda")
    z = t.full((rows + 1, G), 99, dtype=t.uint8, device="cuda") if zeros else None
    q = D.Q4(rows, K, group, dtype, codes.data_ptr(), scales.data_ptr(), z.data_ptr() if zeros else 0)
    wd = w.cuda()
    q.quantize(wd.data_ptr(), ldw, src, stream())
    back = t.full((rows, K + 5), 3.0, dtype=tt(dtype), device="cuda")
    q.dequantize(back.data_ptr(), K + 5, dtype, stream())
    back32 = t.full((rows, K), 3.0, device="cuda")
    q.dequantize(back32.data_ptr(), K, D.FP32, stream())
    t.cuda.synchronize()
    # the formula in numpy fp32, whose divisions are correctly rounded
    v = np.zeros((rows, Kp), np.float32)
    v[:, :K] = w[:, :K].float().numpy()
    v = v.reshape(rows, G, group)
    if zeros:
        lo, hi = np.minimum(v.min(2), np.float32(0)), np.maximum(v.max(2), np.float32(0))
        raw = (hi - lo) / np.float32(15)
    else:
        lo, raw = None, np.abs(v).max(2) / np.float32(7)
    s16 = t.from_numpy(raw).to(tt(dtype))
    s = s16.float().numpy()
    safe = np.where(s > 0, s, np.float32(1))
    zr = np.clip(np.rint(-lo / safe), 0, 15) if zeros else np.full_like(s, 8)
    zr = np.where(s > 0, zr, 8).astype(np.float32)
    qv = np.clip(np.rint(v / safe[:, :, None]) + zr[:, :, None], 0, 15)
    qv = np.where((s > 0)[:, :, None], qv, zr[:, :, None])
    want = D.pack_codes(qv.reshape(rows, Kp).astype(np.uint8))
    assert np.array_equal(codes[:rows].cpu().numpy(), want)
    assert t.equal(scales[:rows].cpu(), s16)
    if zeros:
        assert np.array_equal(z[:rows].cpu().numpy(), zr.astype(np.uint8))
        assert (z[rows] == 99).all()
    assert (codes[rows] == 0xa5).all() and (scales[rows] == 7).all()             # nothing beyond the rows
    values = ((qv - zr[:, :, None]) * s[:, :, None]).reshape(rows, Kp)[:, :K].astype(np.float32)   # exact in fp32
    assert np.array_equal(back32.cpu().numpy(), values)
    assert t.equal(back[:, :K].cpu(), t.from_numpy(values).to(tt(dtype)))
    assert (back[:, K:] == 3).all()


def quantized(w, group, dtype, zeros):
    """codes (as numbers), scales and zero points of a host matrix, from the kernel"""
    t = torch()
    rows, K = w.shape
    G = groups(K, group)
    codes = t.zeros(rows, D.padded_k(K) // 2, dtype=t.uint8, device="cuda")
    scales = t.zeros(rows, G, dtype=tt(dtype), device="cuda")
    z = t.zeros(rows, G, dtype=t.uint8, device="cuda") if zeros else None
    wd = w.cuda()
    D.Q4(rows, K, group, dtype, codes.data_ptr(), scales.data_ptr(), z.data_ptr() if zeros else 0).quantize(
        wd.data_ptr(), K, {t.bfloat16: D.BF16, t.float16: D.FP16, t.float32: D.FP32}[w.dtype], stream())
    return codes.cpu().numpy(), scales.cpu(), None if z is None else z.cpu().numpy()


@pytest.mark.parametrize("src", [D.BF16, D.FP32])
@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_many_ties_and_neighbours_of_ties(src, zeros):
    """Weights at, one step below and one step above the middle of two codes, at scales over the whole range."""
    t = torch()
    rows, K = 240, 128
    w = np.zeros((rows, K), np.float32)
    for r in range(rows):
        s = np.float32(2.0 ** (r - 120)) * np.float32(1 + (r % 7) / 8)
        w[r, 0], w[r, 1] = 7 * s, -7 * s
        mid = (np.arange(2, K) % 14 - 6.5).astype(np.float32) * s
        step = np.arange(2, K) % 3 - 1
        w[r, 2:] = np.where(step < 0, np.nextafter(mid, np.float32(-1e38)), np.where(step > 0, np.nextafter(mid, np.float32(1e38)), mid))
    w = t.from_numpy(w).to(tt(src))
    codes, scales, z = quantized(w, 128, D.BF16, zeros)
    v, s = w.float().numpy(), scales.float().numpy()
    if zeros:
        raw = (np.maximum(v.max(1), np.float32(0)) - np.minimum(v.min(1), np.float32(0))) / np.float32(15)
        zr = np.clip(np.rint(-np.minimum(v.min(1), np.float32(0)) / s[:, 0]), 0, 15).astype(np.float32)
        assert np.array_equal(z[:, 0], zr)
    else:
        raw, zr = np.abs(v).max(1) / np.float32(7), np.full(rows, 8, np.float32)
    assert t.equal(t.from_numpy(raw).bfloat16(), scales[:, 0])
    q = np.clip(np.rint(v / s) + zr[:, None], 0, 15).astype(np.uint8)
    assert np.array_equal(codes, D.pack_codes(q))


def test_quantize_extremes():
    """Scales that are subnormal, beyond their type's range or zero, and quotients far beyond the codes."""
    t = torch()
    w = t.zeros(6, 128)
    w[0, :4] = t.tensor([1e-7, -1e-7, 5e-8, 3e-8])          # fp16: a scale of a few units in the last place
    w[1, :2] = t.tensor([1e-9, -1e-9])                      # rounds to 0
    w[2, :4] = t.tensor([3e38, -3e38, 8e11, -8e11])         # saturates; quotients of 1e33 and 1e7
    w[3, :2] = t.tensor([1e-40, -1e-40])                    # subnormal weights
    w[4, :2] = t.tensor([5e5, -4.6e5])
    codes, scales, _ = quantized(w, 128, D.FP16, False)
    s = np.minimum(np.abs(w.numpy()).max(1) / np.float32(7), np.float32(65504)).astype(np.float16)
    assert np.array_equal(scales[:, 0].numpy(), s)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s[:, None] > 0, np.clip(np.rint(w.numpy() / s[:, None].astype(np.float32)), -8, 7) + 8, 8).astype(np.uint8)
    assert np.array_equal(codes, D.pack_codes(q))


def test_quantize_saturates_a_scale_that_its_type_cannot_hold():
    t = torch()
    w = t.full((1, 128), 3.0e38, device="cuda")
    codes, scales = t.zeros(1, 64, dtype=t.uint8, device="cuda"), t.zeros(1, 1, dtype=t.float16, device="cuda")
    D.Q4(1, 128, 128, D.FP16, codes.data_ptr(), scales.data_ptr()).quantize(w.data_ptr(), 128, D.FP32, stream())
    assert scales.item() == 65504.0 and (codes == 0xff).all()


# ------------------------------------------------------------------ gemv
GEMV = [  # tokens, rows, K, group, zeros
    (1, 1, 1, 32, False), (1, 16, 128, 128, False), (1, 17, 129, 64, True), (2, 100, 1000, 32, True), (1, 4096, 512, 128, True),
    (1, 40, 16384, 128, False), (3, 333, 2052, 64, False), (8, 64, 4096, 128, False), (9, 70, 777, 32, True),
    (16, 130, 1024, 64, True), (17, 200, 640, 128, False), (33, 65, 1536, 32, False), (64, 257, 2048, 128, True),
    (64, 40, 9001, 64, True), (31, 1000, 384, 128, True), (24, 4000, 1100, 64, False), (5, 2100, 700, 32, True),
    (4, 17, 200000, 128, False), (11, 20, 150001, 32, True),   # activations that fit no shared memory
]


@pytest.mark.parametrize("tokens,rows,K,group,zeros", GEMV)
@pytest.mark.parametrize("dtype,out", [(D.BF16, D.BF16), (D.FP16, D.FP32), (D.FP16, D.FP16), (D.BF16, D.FP32)])
def test_gemv_against_its_definition(tokens, rows, K, group, zeros, dtype, out):
    t = torch()
    m = Matrix(rows, K, group, dtype, zeros, seed=tokens * 7 + rows)
    gen = t.Generator().manual_seed(K)
    odd = rows % 2 == 1                                  # rows of x and y off any alignment, or padded ones
    ldx, ldy = K + (1 if odd else 8 - K % 8), rows + 3
    x = t.full((tokens, ldx), float("nan"), dtype=tt(dtype))
    x[:, :K] = t.randn(tokens, K, generator=gen)
    y0 = t.randn(tokens, ldy, generator=gen).to(tt(out))
    xd = x.cuda()
    ref = x[:, :K].double().numpy() @ m.values.T
    mag = np.abs(x[:, :K].double().numpy()) @ np.abs(m.values).T
    for alpha, beta in ((1.0, 0.0), (-0.5, 0.75)):
        y = y0.clone()
        if beta == 0.0:
            y[:, :rows] = float("nan")                   # not read
        yd = y.cuda()
        m.q4().gemv(tokens, xd.data_ptr(), ldx, yd.data_ptr(), ldy, out, alpha, beta, stream())
        got = yd.cpu()
        want = alpha * ref + (beta * y0[:, :rows].double().numpy() if beta else 0.0)
        bound = abs(alpha) * sum_bound(K) * mag + 4 * 2.0 ** -24 * np.abs(want) + U[out] * 1.01 * np.abs(want) + TINY[out]
        err = np.abs(got[:, :rows].double().numpy() - want)
        assert (err <= bound).all(), (err / bound).max()
        assert t.equal(got[:, rows:], y0[:, rows:])      # nothing beside the matrix


def test_gemv_without_products():
    t = torch()
    m = Matrix(70, 256, 64, D.BF16, False, seed=1)
    m.codes.fill_(0)
    for K, alpha in ((256, 0.0), (0, 1.0)):
        for beta in (0.0, 2.0):
            y = t.full((3, 70), float("nan") if beta == 0 else 1.5, device="cuda")
            q = D.Q4(70, K, 64, D.BF16, m.codes.data_ptr(), m.scales.data_ptr())
            q.gemv(3, 0, max(K, 1), y.data_ptr(), 70, D.FP32, alpha, beta, stream())
            assert (y == 1.5 * beta).all()


def test_gemv_keeps_infinities_to_their_token_and_row():
    t = torch()
    m = Matrix(50, 384, 128, D.FP16, True, seed=5)
    x = t.randn(4, 384, generator=t.Generator().manual_seed(1)).half().cuda()
    clean = t.empty(4, 50, device="cuda")
    m.q4().gemv(4, x.data_ptr(), 384, clean.data_ptr(), 50, D.FP32, stream=stream())
    x[1, 100] = float("nan")
    m.scales[7, 1] = float("inf")
    y = t.empty(4, 50, device="cuda")
    m.q4().gemv(4, x.data_ptr(), 384, y.data_ptr(), 50, D.FP32, stream=stream())
    assert t.isnan(y[1]).all()
    rest = [r for r in range(50) if r != 7]
    for token in (0, 2, 3):
        assert t.equal(y[token, rest], clean[token, rest]) and not t.isfinite(y[token, 7])


@pytest.mark.parametrize("dtype", [D.BF16, D.FP16])
def test_gemv_of_infinities_gives_infinities(dtype):
    """inf * 0 is NaN, inf times another weight is inf, and both stay in their token."""
    t = torch()
    m = Matrix(40, 300, 32, dtype, True, seed=15)
    x = t.randn(3, 300, generator=t.Generator().manual_seed(1)).to(tt(dtype))
    x[1, 3], x[2, 290], x[2, 17] = float("inf"), float("-inf"), float("nan")
    y = t.empty(3, 40, device="cuda")
    xd = x.cuda()
    m.q4().gemv(3, xd.data_ptr(), 300, y.data_ptr(), 40, D.FP32, stream=stream())
    y = y.cpu().numpy()
    w = m.values[:, 3]
    assert np.array_equal(np.isnan(y[1]), w == 0) and (y[1][w > 0] == np.inf).all() and (y[1][w < 0] == -np.inf).all()
    assert np.isfinite(y[0]).all() and np.isnan(y[2]).all()


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5])
def test_gemv_at_the_ends_of_the_activations_range(tokens):
    """Tiny, huge and mixed magnitudes within one group of 128, against the bound that the header states."""
    t = torch()
    rows, K = 64, 640
    m = Matrix(rows, K, 128, D.BF16, False, seed=21, spread=1.0)
    gen = t.Generator().manual_seed(tokens)
    x = t.randn(tokens, K, generator=gen) * 2.0 ** t.randint(-30, 30, (tokens, K), generator=gen).float()
    x[:, 128:256] *= 2.0 ** -100
    x[:, 256:384] = 0
    x[:, 384:512] *= 2.0 ** 60
    x = x.bfloat16()
    y = t.empty(tokens, rows, device="cuda")
    xd = x.cuda()
    m.q4().gemv(tokens, xd.data_ptr(), K, y.data_ptr(), rows, D.FP32, stream=stream())
    xs = x.double().numpy()
    top = np.abs(xs).reshape(tokens, -1, 128).max(2).repeat(128, 1)
    ref, mag = xs @ m.values.T, np.abs(xs) @ np.abs(m.values).T
    bound = sum_bound(K) * mag + (top * 2.0 ** -30) @ np.abs(m.values).T
    assert (np.abs(y.cpu().double().numpy() - ref) <= bound).all()


def test_a_row_of_zero_weights_gives_zero():
    t = torch()
    m = Matrix(48, 1024, 64, D.BF16, False, seed=2)
    codes = np.full((48, 1024), 8, np.uint8)
    codes[5, 77] = 9
    m.codes = t.from_numpy(D.pack_codes(codes)).cuda()
    for tokens in (1, 4, 7):
        x = (t.randn(tokens, 1024, generator=t.Generator().manual_seed(3)) + 3).bfloat16().cuda()
        y = t.empty(tokens, 48, device="cuda")
        m.q4().gemv(tokens, x.data_ptr(), 1024, y.data_ptr(), 48, D.FP32, stream=stream())
        assert (y[:, [r for r in range(48) if r != 5]] == 0).all() and (y[:, 5] != 0).all()


def test_check_reports_no_wait_that_gave_up():
    assert D.exo_decode_check() == B.OK


def test_gemv_on_a_side_stream_and_in_a_graph_gives_the_same_bits():
    t = torch()
    m = Matrix(1000, 2048, 64, D.BF16, True, seed=9)
    x = t.randn(5, 2048, generator=t.Generator().manual_seed(3)).bfloat16().cuda()
    y = [t.empty(5, 1000, dtype=t.bfloat16, device="cuda") for _ in range(3)]
    q = m.q4()
    run = lambda out: q.gemv(5, x.data_ptr(), 2048, out.data_ptr(), 1000, D.BF16, stream=stream())  # noqa: E731
    run(y[0])
    t.cuda.synchronize()
    side = t.cuda.Stream()
    with t.cuda.stream(side):
        run(y[1])
    side.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        run(y[2])
    for _ in range(3):
        y[2].zero_()
        graph.replay()
    t.cuda.synchronize()
    assert t.equal(y[0], y[1]) and t.equal(y[0], y[2])


def test_quantize_then_gemv_then_dequantize_in_one_stream():
    """Each kernel may start while its predecessor drains: what a predecessor wrote has to be seen all the same."""
    t = torch()
    rows, K = 2048, 2048
    q_codes, q_scales = t.empty(rows, K // 2, dtype=t.uint8, device="cuda"), t.empty(rows, K // 128, dtype=t.bfloat16, device="cuda")
    q = D.Q4(rows, K, 128, D.BF16, q_codes.data_ptr(), q_scales.data_ptr())
    gen = t.Generator(device="cuda").manual_seed(2)
    x = t.randn(2, K, device="cuda", generator=gen).bfloat16()
    ws = [t.randn(rows, K, device="cuda", generator=gen).bfloat16() for _ in range(6)]
    ys = [t.empty(2, rows, device="cuda") for _ in ws]
    back = [t.empty(rows, K, device="cuda") for _ in ws]
    t.cuda.synchronize()
    for w, y, b in zip(ws, ys, back):
        q.quantize(w.data_ptr(), K, D.BF16, stream())
        q.gemv(2, x.data_ptr(), K, y.data_ptr(), rows, D.FP32, stream=stream())
        q.dequantize(b.data_ptr(), K, D.FP32, stream())
    for y, b in zip(ys, back):
        ref, mag = x.double() @ b.double().t(), x.double().abs() @ b.double().abs().t()
        assert ((y.double() - ref).abs() <= sum_bound(K) * mag).all()


# ------------------------------------------------------------------ mixture of experts
class Layer:
    def __init__(self, H, F, E, shared, k, dtype, group=0, zeros=False, renormalize=1, scale=1.0, seed=0, pad=0, merged=False,
                 max_tokens=64):
        t = torch()
        self.H, self.F, self.E, self.shared, self.k, self.dtype = H, F, E, shared, k, dtype
        self.renormalize, self.scale = renormalize, scale
        gen = t.Generator().manual_seed(seed)
        n = E + shared
        self.ldr = H + pad
        self.router = t.full((E, self.ldr), float("nan")).to(tt(dtype))
        self.router[:, :H] = (t.randn(E, H, generator=gen) * 1.5 * H ** -0.5).to(tt(dtype))
        self.mats, self.vals = {}, {}
        if merged:   # rows of gate and up in turn, expert by expert
            both = self._stack(n * 2 * F, H, group, zeros, pad, gen, seed + 1)
            per = 2 * F
            self.vals["gate"] = both["values"].reshape(n, per, H)[:, :F]
            self.vals["up"] = both["values"].reshape(n, per, H)[:, F:]
            self.mats["gate"] = self._matrix(both, per, 0)
            self.mats["up"] = self._matrix(both, per, F)
            self.keep = [both]
        else:
            self.keep = []
            for i, name in enumerate(("gate", "up")):
                extra = 3 if pad else 0
                m = self._stack(n * (F + extra), H, group, zeros, pad, gen, seed + 1 + i)
                self.vals[name] = m["values"].reshape(n, F + extra, H)[:, :F]
                self.mats[name] = self._matrix(m, F + extra, 0)
                self.keep.append(m)
        m = self._stack(n * H, F, group, zeros, pad, gen, seed + 5)
        self.vals["down"] = m["values"].reshape(n, H, F)
        self.mats["down"] = self._matrix(m, H, 0)
        self.keep.append(m)
        self.router_d = self.router.cuda()
        self.weights = D.MoeWeights(self.router_d.data_ptr(), self.ldr, self.mats["gate"], self.mats["up"], self.mats["down"])
        self.plan = D.MoePlan(D.MoeDesc(H, F, E, shared, k, max_tokens, dtype, group, renormalize, scale))

    def _stack(self, rows, K, group, zeros, pad, gen, seed):
        t = torch()
        if group:
            m = Matrix(rows, K, group, self.dtype, zeros, seed, spread=0.5 * K ** -0.5)
            return {"q4": m, "values": m.values}
        w = t.full((rows, K + pad), float("nan")).to(tt(self.dtype))
        w[:, :K] = (t.randn(rows, K, generator=gen) * K ** -0.5).to(tt(self.dtype))
        return {"w": w.cuda(), "ld": K + pad, "values": w[:, :K].double().numpy()}

    def _matrix(self, m, expert_rows, first):
        if "q4" in m:
            q = m["q4"]
            return D.MoeMatrix(q.codes[first:].data_ptr(), 0, expert_rows, q.scales[first:].data_ptr(),
                               0 if q.zeros is None else q.zeros[first:].data_ptr())
        return D.MoeMatrix(m["w"][first:].data_ptr(), m["ld"], expert_rows, 0, 0)

    def run(self, x, ldx, ldy=None, y=None):
        t = torch()
        T = x.shape[0]
        ldy = ldy or self.H
        y = t.full((T, ldy), 5.0, dtype=tt(self.dtype), device="cuda") if y is None else y
        index = t.full((T, self.k), -7, dtype=t.int32, device="cuda")
        weight = t.full((T, self.k), -7.0, device="cuda")
        self.plan.run(self.weights, T, x.data_ptr(), ldx, y.data_ptr(), ldy, index.data_ptr(), weight.data_ptr(), stream())
        return y, index, weight

    def check(self, x, y, index, weight):
        """x: T x H on the host.  The taken experts have to be a right choice up to the logits' own error."""
        x = x.double().numpy()
        y, index, weight = y.double().cpu().numpy()[:, :self.H], index.cpu().numpy(), weight.double().cpu().numpy()
        r = self.router[:, :self.H].double().numpy()
        logits, lb = x @ r.T, sum_bound(self.H) * (np.abs(x) @ np.abs(r).T)
        for tok in range(len(x)):
            e, took = index[tok], np.zeros(self.E, bool)
            assert ((e >= 0) & (e < self.E)).all() and len(set(e)) == self.k
            took[e] = True
            if not took.all():
                low, high = np.where(took, logits[tok] + lb[tok], np.inf).min(), np.where(took, -np.inf, logits[tok] - lb[tok]).max()
                assert low >= high
            p = np.exp(logits[tok] - logits[tok].max())
            w = p[e] / (p[e].sum() if self.renormalize else p.sum()) * self.scale
            # a logit off by b changes exp by a factor e^b; sums and quotients of at most 520 terms add 2^-14 at most
            assert (np.abs(weight[tok] - w) <= w * (np.expm1(2 * lb[tok].max()) + 2.0 ** -14)).all()
            assert (np.diff(weight[tok]) <= 0).all()
            ref, bound = np.zeros(self.H), np.zeros(self.H)
            for ex, we in list(zip(e, weight[tok])) + [(self.E + s, 1.0) for s in range(self.shared)]:
                g, u = self.vals["gate"][ex] @ x[tok], self.vals["up"][ex] @ x[tok]
                bg = sum_bound(self.H) * (np.abs(self.vals["gate"][ex]) @ np.abs(x[tok]))
                bu = sum_bound(self.H) * (np.abs(self.vals["up"][ex]) @ np.abs(x[tok]))
                silu = g / (1 + np.exp(-g))
                h = we * silu * u
                # |silu'| < 1.1; a few fp32 roundings and expf's; then one rounding to 16 bits
                bh = we * (1.1 * bg * (np.abs(u) + bu) + np.abs(silu) * bu) + np.abs(h) * (16 * 2.0 ** -24 + U[self.dtype]) * 1.01 + TINY[self.dtype]
                d = self.vals["down"][ex]
                ref += d @ h
                bound += np.abs(d) @ bh + sum_bound(self.F) * (np.abs(d) @ np.abs(h))
            n = self.k + self.shared
            bound += np.abs(ref) * U[self.dtype] * 1.01 + TINY[self.dtype] + n * 2.0 ** -20 * np.abs(ref)
            err = np.abs(y[tok] - ref)
            assert (err <= bound).all(), (tok, (err / bound).max())


def tokens(T, H, dtype, seed, pad=0):
    t = torch()
    x = t.full((T, H + pad), float("nan")).to(tt(dtype))
    x[:, :H] = t.randn(T, H, generator=t.Generator().manual_seed(seed)).to(tt(dtype))
    return x


MOE = [  # T, H, F, E, shared, k, group, zeros, pad, merged
    (1, 64, 32, 4, 0, 2, 0, False, 0, False),
    (1, 1, 1, 1, 0, 1, 0, False, 0, False),
    (1, 520, 136, 8, 1, 3, 0, False, 8, False),
    (3, 133, 77, 5, 0, 2, 0, False, 0, False),        # rows off any alignment
    (8, 256, 200, 16, 2, 4, 0, False, 0, True),
    (9, 300, 96, 7, 0, 7, 0, False, 4, True),         # every expert taken; unaligned rows
    (17, 512, 64, 33, 0, 5, 0, False, 0, False),
    (64, 264, 128, 6, 1, 2, 0, False, 0, False),      # many tokens to an expert
    (64, 128, 40, 512, 0, 16, 0, False, 0, False),
    (1, 256, 128, 4, 0, 2, 128, False, 0, False),
    (2, 300, 200, 8, 1, 3, 64, True, 0, False),
    (5, 1000, 130, 6, 0, 2, 32, True, 0, True),
    (12, 384, 256, 20, 0, 4, 128, True, 0, False),
    (64, 160, 96, 5, 1, 2, 32, False, 0, False),
    (33, 2048, 64, 3, 0, 1, 64, False, 0, True),
    (4, 100, 33, 6, 0, 2, 128, True, 0, True),        # one group to a row: rows' scales lie 2 bytes apart
]


@pytest.mark.parametrize("T,H,F,E,shared,k,group,zeros,pad,merged", MOE)
@pytest.mark.parametrize("dtype", [D.BF16, D.FP16])
def test_moe_against_its_definition(T, H, F, E, shared, k, group, zeros, pad, merged, dtype):
    t = torch()
    for renormalize, scale in ((1, 1.0), (0, 2.5)):
        L = Layer(H, F, E, shared, k, dtype, group, zeros, renormalize, scale, seed=T + H, pad=pad, merged=merged, max_tokens=max(T, 2))
        x = tokens(T, H, dtype, T * 31 + H, pad=3 if pad else 0)
        xd = x.cuda()
        y, index, weight = L.run(xd, xd.shape[1], ldy=H + 5)
        assert (y[:, H:] == 5).all()
        L.check(x[:, :H], y, index, weight)
        y2, index2, weight2 = L.run(xd, xd.shape[1], ldy=H + 5)      # the workspace is left as it was found
        assert t.equal(y, y2) and t.equal(index, index2) and t.equal(weight, weight2)


def test_moe_ties_go_to_the_lowest_index():
    t = torch()
    L = Layer(64, 32, 40, 0, 4, D.BF16, seed=3)
    L.router_d.zero_()
    L.router.zero_()
    x = tokens(3, 64, D.BF16, 1)
    xd = x.cuda()
    y, index, weight = L.run(xd, 64)
    assert (index.cpu() == t.arange(4, dtype=t.int32)).all() and (weight == 0.25).all()
    L.check(x, y, index, weight)
    L.router_d[35] = L.router_d[3] = 1.0                 # two equal ones, the largest or the smallest by the token's sign
    _, index, _ = L.run(xd, 64)
    up = x.float().sum(1) > 0
    for tok in range(3):
        assert index[tok].tolist() == ([3, 35, 0, 1] if up[tok] else [0, 1, 2, 4])


def test_moe_all_tokens_to_one_expert():
    t = torch()
    L = Layer(96, 48, 8, 0, 1, D.FP16, seed=4)
    x = tokens(50, 96, D.FP16, 2).abs()
    L.router_d[5] = L.router[5] = 4.0
    xd = x.cuda()
    y, index, weight = L.run(xd, 96)
    assert (index == 5).all() and (weight == 1).all()
    L.check(x, y, index, weight)


def test_moe_fewer_tokens_than_the_plan_and_none():
    t = torch()
    L = Layer(128, 64, 12, 1, 3, D.BF16, seed=6, max_tokens=64)
    for T in (64, 1, 20, 7):
        x = tokens(T, 128, D.BF16, T)
        xd = x.cuda()
        L.check(x, *L.run(xd, 128))
    y = t.full((1, 128), 5.0, dtype=t.bfloat16, device="cuda")
    L.plan.run(L.weights, 0, 0, 128, 0, 128)
    L.plan.run(L.weights, 1, tokens(1, 128, D.BF16, 1).cuda().data_ptr(), 128, y.data_ptr(), 128, stream=stream())   # no index, no weight
    assert not (y == 5).all()


def test_moe_keeps_nan_to_its_token_and_an_untaken_expert_out():
    t = torch()
    L = Layer(128, 64, 6, 0, 2, D.BF16, seed=8)
    x = tokens(5, 128, D.BF16, 3)
    xd = x.cuda()
    y, index, _ = L.run(xd, 128)
    xd[2, 17] = float("nan")
    used = set(index[[0, 1, 3, 4]].flatten().tolist())
    y2, index2, weight2 = L.run(xd, 128)
    assert t.isnan(y2[2]).all() and t.isnan(weight2[2]).all()
    assert ((index2 >= 0) & (index2 < 6)).all()
    keep = [0, 1, 3, 4]
    assert t.equal(index[keep], index2[keep]) and t.equal(y[keep], y2[keep])
    L2 = Layer(128, 64, 6, 0, 2, D.BF16, seed=8)
    for e in set(range(6)) - set(index.flatten().tolist()):
        L2.keep[0]["w"][e * 64:(e + 1) * 64] = float("nan")
    xd = x.cuda()
    assert t.equal(L2.run(xd, 128)[0], y) and used


def test_moe_captured_in_a_graph_and_on_a_side_stream():
    t = torch()
    L = Layer(512, 256, 16, 1, 4, D.FP16, group=64, zeros=True, seed=10)
    x = tokens(6, 512, D.FP16, 9).cuda()
    want, index, weight = L.run(x, 512)
    t.cuda.synchronize()
    side = t.cuda.Stream()
    with t.cuda.stream(side):
        got, _, _ = L.run(x, 512)
    side.synchronize()
    assert t.equal(want, got)
    y = t.zeros(6, 512, dtype=t.float16, device="cuda")
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        L.plan.run(L.weights, 6, x.data_ptr(), 512, y.data_ptr(), 512, stream=stream())
        L.plan.run(L.weights, 6, x.data_ptr(), 512, y.data_ptr(), 512, stream=stream())
    for _ in range(3):
        y.zero_()
        graph.replay()
    t.cuda.synchronize()
    assert t.equal(want, y)


def test_moe_runs_in_a_row_with_changing_inputs():
    """Each run's first kernel may start while the last one drains; they share the workspace."""
    t = torch()
    L = Layer(256, 128, 32, 0, 6, D.BF16, seed=12)
    xs = [tokens(T, 256, D.BF16, T).cuda() for T in (1, 40, 3, 64, 2, 9)]
    first = [L.run(x, 256) for x in xs]
    again = [L.run(x, 256) for x in xs for _ in range(1)]
    alone = []
    for x in xs:
        alone.append(L.run(x, 256))
        t.cuda.synchronize()
    for a, b, c in zip(first, again, alone):
        for u, v, w in zip(a, b, c):
            assert t.equal(u, v) and t.equal(u, w)


def test_moe_refuses_bad_arguments():
    t = torch()
    L = Layer(64, 32, 4, 0, 2, D.BF16, seed=1, max_tokens=4)
    buf = t.zeros(1 << 16, dtype=t.uint8, device="cuda").data_ptr()
    run = lambda w=L.weights, T=1, x=buf, ldx=64, y=buf + 8192, ldy=64, i=0, wt=0: D.exo_moe_run(L.plan.handle, w, T, x, ldx, y, ldy, i, wt)  # noqa: E731
    assert run(w=None) == B.ERR_NULL and run(x=0) == B.ERR_NULL and run(y=0) == B.ERR_NULL
    assert run(T=5) == B.ERR_INVALID_ARG and run(T=-1) == B.ERR_INVALID_ARG
    assert run(ldx=63) == B.ERR_INVALID_ARG and run(ldy=63) == B.ERR_INVALID_ARG
    assert run(x=buf + 1) == B.ERR_ALIGNMENT and run(i=buf + 2) == B.ERR_ALIGNMENT and run(wt=buf + 2) == B.ERR_ALIGNMENT

    def changed(which, **kw):
        mats = {n: D.MoeMatrix(*[getattr(L.mats[n], f) for f, _ in D.MoeMatrix._fields_]) for n in L.mats}
        for name, value in kw.items():
            setattr(mats[which], name, value)
        return D.MoeWeights(L.router_d.data_ptr(), 64, mats["gate"], mats["up"], mats["down"])
    for which, K, rows in (("gate", 64, 32), ("up", 64, 32), ("down", 32, 64)):
        assert run(w=changed(which, w=0)) == B.ERR_NULL
        assert run(w=changed(which, ld=K - 1)) == B.ERR_INVALID_ARG
        assert run(w=changed(which, expert_rows=rows - 1)) == B.ERR_INVALID_ARG
        assert run(w=changed(which, scales=buf)) == B.ERR_INVALID_ARG
        assert run(w=changed(which, w=buf + 1)) == B.ERR_ALIGNMENT
    assert run(w=D.MoeWeights(0, 64, L.mats["gate"], L.mats["up"], L.mats["down"])) == B.ERR_NULL
    assert run(w=D.MoeWeights(buf, 63, L.mats["gate"], L.mats["up"], L.mats["down"])) == B.ERR_INVALID_ARG
    Q = Layer(64, 32, 4, 0, 2, D.BF16, group=32, seed=1, max_tokens=4)
    bad = D.MoeWeights(Q.router_d.data_ptr(), 64, D.MoeMatrix(Q.mats["gate"].w, 0, 32, 0, 0), Q.mats["up"], Q.mats["down"])
    assert D.exo_moe_run(Q.plan.handle, bad, 1, buf, 64, buf + 8192, 64) == B.ERR_NULL
    bad = D.MoeWeights(Q.router_d.data_ptr(), 64, D.MoeMatrix(Q.mats["gate"].w + 8, 0, 32, Q.mats["gate"].scales, 0), Q.mats["up"], Q.mats["down"])
    assert D.exo_moe_run(Q.plan.handle, bad, 1, buf, 64, buf + 8192, 64) == B.ERR_ALIGNMENT
    assert Q.plan.workspace_bytes() >= 4 * 2 * 32 * 2
    t.cuda.synchronize()


# ------------------------------------------------------------------ all of them together
@pytest.mark.parametrize("tokens", [1, 6])
def test_decode_layer_example(tokens):
    """The tokens' projection from 4 bits is the prompt's GEMM on the dequantised weights: W's values are exact in fp32 but
    rounded to bf16 for the GEMM (2^-8 each), the sums are fp32, and both results are rounded to bf16."""
    from examples import decode_layer
    t = torch()
    h, by_prompt, y, taken = decode_layer.run(tokens, hidden=768, inner=320, experts=12, top_k=3, prompt=96, seed=tokens)
    a, b = h.double(), by_prompt.double()
    assert ((a - b).norm() / b.norm()).item() <= 3 * 2.0 ** -8
    assert t.isfinite(y).all() and ((taken >= 0) & (taken < 12)).all()


# ------------------------------------------------------------------ one or two tokens and a large matrix: integer products
class LargeMatrix:
    """A 4-bit matrix of random codes made on the device; ``values`` are its weights in 64 bits."""

    def __init__(self, rows, K, group, dtype, zeros, seed):
        t = torch()
        gen = t.Generator(device="cuda").manual_seed(seed)
        self.rows, self.K, self.group, self.dtype = rows, K, group, dtype
        kp = D.padded_k(K)
        words = t.randint(-2 ** 31, 2 ** 31, (rows, kp // 8), generator=gen, device="cuda", dtype=t.int64).int()
        G = groups(K, group)
        self.codes = words
        self.scales = ((t.rand(rows, G, generator=gen, device="cuda") + 0.25) * 0.02).to(tt(dtype))
        self.scales[:, (K + group - 1) // group:] = float("nan")
        self.zeros = t.randint(0, 16, (rows, G), generator=gen, device="cuda", dtype=t.uint8) if zeros else None
        # weight 128 b + 32 j + 8 t + i is nibble i / 2 + 4 (i % 2) of word 16 b + 4 t + j
        w = words.view(rows, kp // 128, 4, 4).permute(0, 1, 3, 2)
        codes = t.empty(rows, kp // 128, 4, 4, 8, device="cuda", dtype=t.uint8)
        for i in range(8):
            codes[..., i] = (w >> (4 * (i // 2 + 4 * (i % 2)))) & 15
        at = t.arange(K, device="cuda") // group
        zero = self.zeros.double()[:, at] if zeros else 8.0
        self.values = (codes.view(rows, kp)[:, :K].double() - zero) * self.scales.double()[:, at]

    def gemv(self, x, y, alpha=1.0, beta=0.0):
        q = D.Q4(self.rows, self.K, self.group, self.dtype, self.codes.data_ptr(), self.scales.data_ptr(),
                 0 if self.zeros is None else self.zeros.data_ptr())
        out = {v: k for k, v in ((k, tt(k)) for k in (D.BF16, D.FP16, D.FP32))}[y.dtype]
        q.gemv(x.shape[0], x.data_ptr(), x.stride(0), y.data_ptr(), y.stride(0), out, alpha, beta, stream())

    def bound(self, x):
        """What sums in fp32 and activations within 2^-30 of the largest of their 128 may be off by."""
        t = torch()
        xs = t.zeros(x.shape[0], D.padded_k(self.K), device="cuda", dtype=t.float64)
        xs[:, :self.K] = x[:, :self.K].double().abs()
        top = xs.view(x.shape[0], -1, 128).amax(2).repeat_interleave(128, 1)[:, :self.K]
        return (sum_bound(self.K) * xs[:, :self.K] + 2.0 ** -30 * top) @ self.values.abs().T


LARGE = [  # tokens, rows, K, group, zeros: 38 MB of weights or more, few and many rows, odd ends
    (1, 4000, 20010, 128, False), (2, 18961, 4100, 32, True), (2, 1297, 60001, 64, False), (1, 606500, 100, 128, True),
    (1, 9001, 9001, 64, True), (2, 32768, 2560, 32, False)]


@pytest.mark.parametrize("tokens,rows,K,group,zeros", LARGE)
@pytest.mark.parametrize("dtype,out", [(D.BF16, D.FP32), (D.FP16, D.FP16)])
def test_gemv_of_large_matrices_against_its_definition(tokens, rows, K, group, zeros, dtype, out):
    t = torch()
    m = LargeMatrix(rows, K, group, dtype, zeros, seed=rows)
    gen = t.Generator(device="cuda").manual_seed(K)
    x = t.randn(tokens, K + K % 2, generator=gen, device="cuda").to(tt(dtype))
    x[:, K:] = float("nan")
    ref, bound = x[:, :K].double() @ m.values.T, m.bound(x)
    y0 = t.randn(tokens, rows + 3, generator=gen, device="cuda").to(tt(out))
    for alpha, beta in ((1.0, 0.0), (-0.5, 0.75)):
        y = y0.clone()
        if beta == 0.0:
            y[:, :rows] = float("nan")
        m.gemv(x, y, alpha, beta)
        want = alpha * ref + (beta * y0[:, :rows].double() if beta else 0.0)
        off = (y[:, :rows].double() - want).abs()
        allowed = abs(alpha) * bound + (4 * 2.0 ** -24 + U[out] * 1.01) * want.abs() + TINY[out]
        assert bool((off <= allowed).all()), float((off / allowed).max())
        assert t.equal(y[:, rows:], y0[:, rows:])
        again = y0.clone()
        m.gemv(x, again, alpha, beta)
        assert t.equal(again[:, :rows], y[:, :rows])


def test_gemv_of_large_matrices_at_the_ends_of_the_activations_range():
    t = torch()
    m = LargeMatrix(9000, 9000, 128, D.BF16, False, seed=3)
    gen = t.Generator(device="cuda").manual_seed(4)
    x = t.randn(2, 9000, generator=gen, device="cuda") * 2.0 ** t.randint(-30, 30, (2, 9000), generator=gen, device="cuda").float()
    x[:, 128:256] *= 2.0 ** -100
    x[:, 256:384] = 0
    x[:, 384:512] *= 2.0 ** 60
    x = x.bfloat16()
    y = t.empty(2, 9000, device="cuda")
    m.gemv(x, y)
    ref = x.double() @ m.values.T
    assert bool(((y.double() - ref).abs() <= m.bound(x) + (4 * 2.0 ** -24 + U[D.FP32] * 1.01) * ref.abs()).all())


@pytest.mark.parametrize("dtype", [D.BF16, D.FP16])
def test_gemv_of_large_matrices_keeps_infinities_to_their_token_and_row(dtype):
    t = torch()
    m = LargeMatrix(4000, 20010, 32, dtype, True, seed=6)
    x = t.randn(2, 20010, generator=t.Generator(device="cuda").manual_seed(7), device="cuda").to(tt(dtype))
    clean = t.empty(2, 4000, device="cuda")
    m.gemv(x, clean)
    x[1, 20009] = float("inf")
    y = t.empty(2, 4000, device="cuda")
    m.gemv(x, y)
    w = m.values[:, 20009]
    assert t.equal(y[0], clean[0]) and t.equal(t.isnan(y[1]), w == 0)
    assert bool((y[1][w > 0] == float("inf")).all()) and bool((y[1][w < 0] == float("-inf")).all())
    m.scales[7, 3] = float("inf")
    m.gemv(x, y)
    rest = t.arange(4000, device="cuda") != 7
    assert t.equal(y[0][rest], clean[0][rest]) and not t.isfinite(y[0, 7])


# ------------------------------------------------------------------ launches that no larger one has prepared
FIRST = [  # T, H, F, E, shared, k, group: around the token counts at which the kernels' shared memory passes 48 KB
    (20, 160, 96, 5, 0, 2, 0), (28, 160, 96, 5, 0, 2, 0), (36, 160, 96, 5, 1, 2, 0), (40, 160, 96, 5, 0, 2, 32), (48, 160, 96, 5, 0, 2, 0),
    (64, 133, 77, 5, 0, 2, 0), (28, 4096, 64, 5, 0, 2, 0), (36, 4096, 64, 5, 1, 2, 0), (40, 1100, 64, 5, 0, 2, 0)]


@pytest.mark.parametrize("T,H,F,E,shared,k,group", FIRST)
def test_moe_of_any_token_count(T, H, F, E, shared, k, group):
    L = Layer(H, F, E, shared, k, D.BF16, group, False, 1, 1.0, seed=T + H, max_tokens=T)
    x = tokens(T, H, D.BF16, T)
    y, index, weight = L.run(x.cuda(), H, ldy=H)
    L.check(x, y, index, weight)


@pytest.mark.parametrize("case", FIRST, ids=str)
def test_moe_as_a_process_first_call(case):
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    code = "import sys; sys.path[:0] = %r; import test_decode_gpu as m; m.test_moe_of_any_token_count(*%r)" % ([here, os.path.dirname(here)], case)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# ------------------------------------------------------------------ a plan's first run
def test_moe_plan_made_while_the_default_stream_is_busy_runs_on_another_one():
    """A new plan's workspace is clear when it is returned, in whatever order streams get to their work."""
    t = torch()
    T, H, F, E, k = 20, 512, 100, 16, 4
    L = Layer(H, F, E, 0, k, D.FP16, seed=30, max_tokens=T)
    x = tokens(T, H, D.FP16, 31).cuda()
    want, index, weight = L.run(x, H)
    a = t.randn(8192, 8192, device="cuda", dtype=t.bfloat16)
    got = t.zeros(T, H, dtype=t.float16, device="cuda")
    side = t.cuda.Stream()
    a @ a
    t.cuda.synchronize()
    for _ in range(3):
        junk = t.full((L.plan.workspace_bytes(),), 0xff, dtype=t.uint8, device="cuda")   # what the new plan's memory may have held
        t.cuda.synchronize()
        del junk
        t.cuda.empty_cache()
        for _ in range(60):                              # some 40 ms of work
            a @ a
        with D.MoePlan(D.MoeDesc(H, F, E, 0, k, T, D.FP16)) as plan:
            with t.cuda.stream(side):
                plan.run(L.weights, T, x.data_ptr(), H, got.data_ptr(), H, stream=stream())
            side.synchronize()
        t.cuda.synchronize()
        assert t.equal(got, want)


# ------------------------------------------------------------------ large inner activations
def one_expert(H, F, dtype, gate, up, down):
    """A layer of one expert with constant gate and up weights; its weight is 1."""
    L = Layer(H, F, 1, 0, 1, dtype, seed=40, max_tokens=8)
    L.keep[0]["w"].fill_(gate)
    L.keep[1]["w"].fill_(up)
    L.keep[2]["w"].copy_(down)
    return L


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("sign", [1, -1])
def test_moe_inner_activations_beyond_the_largest_fp16_number(T, sign):
    """silu(256) * 273.5 = 70016 = 65504 + 4512: representable as two parts, so that only sums and y's rounding are left."""
    t = torch()
    H, F = 16, 40
    d = (t.randn(H, F, generator=t.Generator().manual_seed(1)) * 0.01).half()
    L = one_expert(H, F, D.FP16, 16.0, 17.09375 * sign, d.cuda())
    x = t.ones(T, H, dtype=t.float16, device="cuda")
    y, _, weight = L.run(x, H)
    assert (weight == 1).all()
    ref, mag = d.double().sum(1) * 70016 * sign, d.double().abs().sum(1) * 70016
    bound = sum_bound(F) * mag + U[D.FP16] * 1.01 * ref.abs() + TINY[D.FP16]
    assert bool(((y.cpu().double() - ref).abs() <= bound).all())


@pytest.mark.parametrize("T", [1, 4, 5])
@pytest.mark.parametrize("dtype,x,gate", [(D.FP16, 4.0, 1024.0), (D.BF16, 1.0e25, 1.0e8)])
def test_moe_inner_activations_beyond_their_type_are_infinite(T, dtype, x, gate):
    """(fp16: 2^16 squared; bf16: beyond fp32 as well.)  An infinity keeps its sign through positive and negative weights."""
    t = torch()
    H, F = 16, 40
    d = t.full((H, F), 2.0 ** -20)
    d[H // 2:] = -2.0 ** -20
    L = one_expert(H, F, dtype, gate, gate, d.to(tt(dtype)).cuda())
    y, _, _ = L.run(t.full((T, H), x, dtype=tt(dtype), device="cuda"), H)
    assert (y[:, :H // 2] == float("inf")).all() and (y[:, H // 2:] == -float("inf")).all()


# ------------------------------------------------------------------ integer products over all of bf16's range
def scaled(m, exponent):
    """m with its scales (and so its values) times 2^exponent, a power that bf16 scales of 0.005 and more take exactly."""
    m.scales = (m.scales.float() * 2.0 ** exponent).to(m.scales.dtype)
    m.values = m.values * 2.0 ** exponent
    return m


# a result below the smallest normal number is off by half the last subnormal bit for each of an fp32 sum's roundings: four columns of
# digits in steps of 128, and the sums of warps and CTAs
def tiny_bound(K):
    return (K / 32 + 64) * 2.0 ** -150


@pytest.mark.parametrize("tokens", [1, 2, 3])
@pytest.mark.parametrize("group,zeros", [(128, False), (32, True)])
@pytest.mark.parametrize("x_exp,s_exp", [(-83, -43), (-60, -60), (-100, -20), (-123, 0), (-129, 20), (60, 50), (-20, 118), (110, -100)])
def test_gemv_of_large_matrices_at_any_magnitude(tokens, group, zeros, x_exp, s_exp):
    t = torch()
    m = scaled(LargeMatrix(9000, 9000, group, D.BF16, zeros, seed=50), s_exp)
    x = (t.randn(tokens, 9000, generator=t.Generator(device="cuda").manual_seed(51), device="cuda", dtype=t.float64) * 2.0 ** x_exp).bfloat16()
    y = t.empty(tokens, 9000, device="cuda")
    m.gemv(x, y)
    ref = x.double() @ m.values.T
    allowed = m.bound(x) + (4 * 2.0 ** -24 + U[D.FP32] * 1.01) * ref.abs() + tiny_bound(9000)
    off = (y.double() - ref).abs()
    assert bool(t.isfinite(y).all()) and bool((off <= allowed).all()), float((off / allowed).max())


@pytest.mark.parametrize("tokens", [1, 2, 3])
def test_gemv_of_large_matrices_up_to_the_largest_float(tokens):
    """130 = 33 * 4 - 2: the second digit is -128 where the first is 33, and its sum overflows before the result does."""
    t = torch()
    m = LargeMatrix(9000, 9000, 64, D.BF16, True, seed=52)
    m.codes.fill_(-1)
    m.zeros.zero_()
    m.scales[:, :] = m.scales[:, :1].float() * 2.0 ** 60
    m.values = (15 * m.scales[:, :1].double()).expand(-1, 9000)
    top = 0.8 * 3.4e38 / float(m.values[:, 0].max() * 9000)
    x = t.full((tokens, 9000), 130 * 2.0 ** np.floor(np.log2(top / 130)), device="cuda").bfloat16()
    y = t.empty(tokens, 9000, device="cuda")
    m.gemv(x, y)
    ref = x.double() @ m.values.T
    assert float(ref.max()) > 1.0e38
    assert bool(((y.double() - ref).abs() <= m.bound(x) + (4 * 2.0 ** -24 + U[D.FP32] * 1.01) * ref.abs()).all())


@pytest.mark.parametrize("tokens", [1, 2, 3])
def test_gemv_of_large_matrices_of_zero_weights_gives_zero(tokens):
    t = torch()
    m = scaled(LargeMatrix(9000, 9000, 128, D.BF16, False, seed=53), 100)
    m.codes.fill_(-0x77777778)                           # 0x88888888
    x = (t.randn(tokens, 9000, generator=t.Generator(device="cuda").manual_seed(54), device="cuda") * 2.0 ** 120).bfloat16()
    y = t.empty(tokens, 9000, device="cuda")
    m.gemv(x, y)
    assert bool((y == 0).all())


# ------------------------------------------------------------------ how inner activations are held
def cancelling_layer(T, H, F, E, k, dtype, group, pad):
    """Neighbouring inner values differ by one step of `dtype` and meet weights of opposite sign: y is small, and what rounds an
    inner activation once to `dtype` shows."""
    t = torch()
    L = Layer(H, F, E, 0, k, dtype, group, False, seed=60, pad=pad, max_tokens=T)
    step = 1 + 2 * U[dtype]
    if group:
        for name, m, factor in (("gate", L.keep[0]["q4"], 1.0), ("up", L.keep[1]["q4"], step)):
            m.codes[1::2] = m.codes[0::2]
            old = m.scales.clone()
            m.scales[1::2] = (m.scales[0::2].float() * factor).to(m.scales.dtype)
            at = np.arange(H) // group
            codes = m.values[0::2] / old[0::2].double().cpu().numpy()[:, at]
            m.values[1::2] = codes * m.scales[1::2].double().cpu().numpy()[:, at]
            L.vals[name] = m.values.reshape(E, F, H)
        m = L.keep[2]["q4"]
        c = np.random.default_rng(61).integers(1, 16, (E * H, F), dtype=np.uint8)
        c[:, 1::2] = 16 - c[:, 0::2]
        m.codes.copy_(t.from_numpy(D.pack_codes(c)))
        m.values = (c.astype(np.float64) - 8) * m.scales.double().cpu().numpy()[:, np.arange(F) // group]
        L.vals["down"] = m.values.reshape(E, H, F)
    else:
        for name, keep, factor in (("gate", L.keep[0], 1.0), ("up", L.keep[1], step)):
            w = keep["w"].view(E, -1, keep["ld"])
            w[:, 1:F:2] = (w[:, 0:F:2].float() * factor).to(w.dtype)
            L.vals[name] = w[:, :F, :H].double().cpu().numpy()
        w = L.keep[2]["w"]
        w[:, 1:F:2] = -w[:, 0:F:2]
        L.vals["down"] = w[:, :F].double().cpu().numpy().reshape(E, H, F)
    return L


@pytest.mark.parametrize("dtype", [D.BF16, D.FP16])
@pytest.mark.parametrize("group,pad", [(0, 0), (0, 1), (32, 0)])
@pytest.mark.parametrize("T,E,k", [(1, 8, 2), (4, 8, 2), (6, 24, 2), (12, 40, 3), (20, 40, 2), (64, 256, 2)])
def test_moe_holds_the_inner_activations_of_few_tokens_in_two_parts(T, E, k, group, pad, dtype):
    """Each token has one channel, so that gate and up are exact.  An inner activation is then off by a few roundings of fp32 and, where its
    expert has up to four tokens, by the rounding of the second part: U * U of it."""
    t = torch()
    H, F = 64, 64
    L = cancelling_layer(T, H, F, E, k, dtype, group, pad)
    x = t.zeros(T, H, dtype=tt(dtype))
    x[t.arange(T), (t.arange(T) * 7) % H] = 4.0
    y, index, weight = L.run(x.cuda(), H)
    y, index, weight, xs = y.double().cpu().numpy(), index.cpu().numpy(), weight.double().cpu().numpy(), x.double().numpy()
    count = np.bincount(index.reshape(-1), minlength=E)
    seen = 0
    for tok in range(T):
        ref, once, bound = np.zeros(H), np.zeros(H), np.zeros(H)
        for e, we in zip(index[tok], weight[tok]):
            g, u, d = L.vals["gate"][e] @ xs[tok], L.vals["up"][e] @ xs[tok], L.vals["down"][e]
            h = we * g / (1 + np.exp(-g)) * u
            part = U[dtype] ** 2 if count[e] <= 4 else U[dtype]
            ref += d @ h
            once += d @ t.from_numpy(h).to(tt(dtype)).double().numpy()
            bound += np.abs(d) @ (np.abs(h) * (16 * 2.0 ** -24 + part * 1.01) + TINY[dtype]) + sum_bound(F) * (np.abs(d) @ np.abs(h))
        bound += np.abs(ref) * (U[dtype] * 1.01 + k * 2.0 ** -20) + TINY[dtype]
        assert (np.abs(y[tok] - ref) <= bound).all(), (tok, (np.abs(y[tok] - ref) / bound).max())
        if (count[index[tok]] <= 4).all():
            seen += 1
            assert (np.abs(once - ref) > bound).any()    # one part would show
    assert seen > 0


# ------------------------------------------------------------------ bounded waits
@pytest.mark.parametrize("tokens,rows,K,group", [(1, 9000, 9000, 128), (5, 2100, 4100, 64), (24, 16384, 1024, 32)])
def test_gemv_reports_a_wait_that_runs_out_and_recovers(tokens, rows, K, group):
    """The first warp issues no copies and waits 20 ms for them: an error status, no trap, and the next call is a good one."""
    t = torch()
    m = LargeMatrix(rows, K, group, D.BF16, True, seed=70)
    x = t.randn(tokens, K, generator=t.Generator(device="cuda").manual_seed(71), device="cuda").bfloat16()
    good, y = t.empty(tokens, rows, device="cuda"), t.empty(tokens, rows, device="cuda")
    m.gemv(x, good)
    assert D.exo_decode_check() == B.OK
    assert D.exo_decode_debug_set(20, 1) == B.OK
    m.gemv(x, y)
    assert D.exo_decode_check() == B.ERR_DEVICE_TIMEOUT
    assert D.exo_decode_check() == B.OK                  # said once
    m.gemv(x, y)
    assert D.exo_decode_check() == B.OK and t.equal(y, good)


@pytest.mark.parametrize("skip", [1, 2])
@pytest.mark.parametrize("T,group", [(2, 0), (12, 0), (40, 0), (2, 128), (20, 32)])
def test_moe_reports_a_wait_that_runs_out_and_recovers(T, group, skip):
    t = torch()
    L = Layer(512, 384, 16, 1, 4, D.BF16, group=group, seed=72, max_tokens=T)
    x = tokens(T, 512, D.BF16, 73).cuda()
    good = L.run(x, 512)
    assert D.exo_decode_check() == B.OK
    assert D.exo_decode_debug_set(20, skip) == B.OK
    L.run(x, 512)
    assert D.exo_decode_check() == B.ERR_DEVICE_TIMEOUT
    again = L.run(x, 512)
    assert D.exo_decode_check() == B.OK and all(t.equal(a, b) for a, b in zip(good, again))


# ------------------------------------------------------------------ rings in use: units beyond the warps, pieces beyond the stages
STEADY = [  # tokens, rows, K, group, zeros: 25000 x 4100 has more units than warps, 16384 x 8192 more pieces than stages as well
    (3, 25000, 4100, 32, True), (3, 16384, 8192, 128, False), (8, 25000, 4100, 64, False), (8, 16384, 8192, 32, True), (9, 25000, 4100, 128, True),
    (24, 16384, 8192, 128, False), (24, 25000, 4100, 64, True), (24, 16384, 8192, 32, False), (40, 16384, 8192, 64, True), (40, 25000, 4100, 32, False),
    (64, 16384, 8192, 128, True), (64, 16384, 8192, 32, False), (64, 25000, 4100, 64, True),
    (32, 4096, 4096, 128, False), (64, 4096, 4096, 64, False), (57, 4096, 4096, 32, True)]   # four tiles of eight tokens to a CTA


@pytest.mark.parametrize("tokens,rows,K,group,zeros", STEADY)
@pytest.mark.parametrize("dtype,out", [(D.BF16, D.FP32), (D.FP16, D.FP16)])
def test_gemv_of_several_tokens_and_large_matrices_against_its_definition(tokens, rows, K, group, zeros, dtype, out):
    t = torch()
    m = LargeMatrix(rows, K, group, dtype, zeros, seed=tokens + rows)
    x = t.randn(tokens, K, generator=t.Generator(device="cuda").manual_seed(K), device="cuda").to(tt(dtype))
    y = t.full((tokens, rows + 1), 3.0, device="cuda").to(tt(out))
    m.gemv(x, y[:, :rows])
    ref = x.double() @ m.values.T
    allowed = sum_bound(K) * (x.double().abs() @ m.values.abs().T) + U[out] * 1.01 * ref.abs() + TINY[out]
    off = (y[:, :rows].double() - ref).abs()
    assert bool((off <= allowed).all()), float((off / allowed).max())
    assert bool((y[:, rows:] == 3).all())


class LargeLayer:
    """A layer whose weights are made, and whose definition is evaluated, on the device."""

    def __init__(self, H, F, E, shared, k, dtype, group, zeros, T, seed):
        t = torch()
        self.H, self.F, self.E, self.shared, self.k, self.dtype = H, F, E, shared, k, dtype
        gen = t.Generator(device="cuda").manual_seed(seed)
        n = E + shared
        self.router = (t.randn(E, H, generator=gen, device="cuda") * 1.5 * H ** -0.5).to(tt(dtype))
        self.vals, self.keep, mats = {}, [], []
        for i, (name, rows, K) in enumerate((("gate", F, H), ("up", F, H), ("down", H, F))):
            if group:
                m = scaled(LargeMatrix(n * rows, K, group, dtype, zeros, seed + 1 + i), -int(np.log2(K) / 2))   # weights of about K^-1/2 / 10
                self.vals[name] = m.values.view(n, rows, K)
                mats.append(D.MoeMatrix(m.codes.data_ptr(), 0, rows, m.scales.data_ptr(), 0 if m.zeros is None else m.zeros.data_ptr()))
            else:
                m = (t.randn(n * rows, K, generator=gen, device="cuda") * K ** -0.5).to(tt(dtype))
                self.vals[name] = m.double().view(n, rows, K)
                mats.append(D.MoeMatrix(m.data_ptr(), K, rows, 0, 0))
            self.keep.append(m)
        self.weights = D.MoeWeights(self.router.data_ptr(), H, *mats)
        self.plan = D.MoePlan(D.MoeDesc(H, F, E, shared, k, T, dtype, group))

    def run(self, x):
        t = torch()
        T = x.shape[0]
        y = t.empty(T, self.H, dtype=tt(self.dtype), device="cuda")
        index, weight = t.empty(T, self.k, dtype=t.int32, device="cuda"), t.empty(T, self.k, device="cuda")
        self.plan.run(self.weights, T, x.data_ptr(), self.H, y.data_ptr(), self.H, index.data_ptr(), weight.data_ptr(), stream())
        return y, index, weight

    def check(self, x, y, index, weight):
        """As Layer.check; the inner activations of experts of up to four tokens are held in two parts."""
        t = torch()
        T, x, at = x.shape[0], x.double(), index.long()
        r = self.router.double()
        logits, lb = x @ r.T, sum_bound(self.H) * (x.abs() @ r.abs().T)
        took = t.zeros(T, self.E, dtype=t.bool, device="cuda").scatter_(1, at, True)
        assert bool((took.sum(1) == self.k).all())
        inf = float("inf")
        assert bool((t.where(took, logits + lb, inf).amin(1) >= t.where(took, -inf, logits - lb).amax(1)).all())
        p = t.exp(logits - logits.amax(1, keepdim=True)).gather(1, at)
        w = p / p.sum(1, keepdim=True)
        assert bool(((weight.double() - w).abs() <= w * (t.expm1(2 * lb.amax(1, keepdim=True)) + 2.0 ** -14)).all())
        part = t.zeros(T, self.E + self.shared, device="cuda", dtype=t.float64)
        part[:, self.E:] = 1
        part[:, :self.E].scatter_(1, at, weight.double())
        ref, bound = t.zeros(T, self.H, device="cuda", dtype=t.float64), t.zeros(T, self.H, device="cuda", dtype=t.float64)
        for e in range(self.E + self.shared):
            rows = part[:, e].nonzero()[:, 0]
            if len(rows) == 0:
                continue
            a, we = x[rows], part[rows, e][:, None]
            gate, up, down = (self.vals[name][e] for name in ("gate", "up", "down"))
            g, u = a @ gate.T, a @ up.T
            bg, bu = sum_bound(self.H) * (a.abs() @ gate.abs().T), sum_bound(self.H) * (a.abs() @ up.abs().T)
            silu = g / (1 + t.exp(-g))
            h = we * silu * u
            held = U[self.dtype] ** 2 if len(rows) <= 4 else U[self.dtype]
            bh = we * (1.1 * bg * (u.abs() + bu) + silu.abs() * bu) + h.abs() * (16 * 2.0 ** -24 + held) * 1.01 + TINY[self.dtype]
            ref[rows] += h @ down.T
            bound[rows] += bh @ down.abs().T + sum_bound(self.F) * (h.abs() @ down.abs().T)
        bound += ref.abs() * (U[self.dtype] * 1.01 + (self.k + self.shared) * 2.0 ** -20) + TINY[self.dtype]
        off = (y.double() - ref).abs()
        assert bool((off <= bound).all()), float((off / bound).max())


@pytest.mark.parametrize("T", [1, 4, 8, 16, 64])
@pytest.mark.parametrize("group,zeros,dtype", [(0, False, D.BF16), (0, False, D.FP16), (128, False, D.BF16), (64, True, D.FP16), (32, True, D.BF16)])
def test_moe_of_many_items_against_its_definition(T, group, zeros, dtype):
    """32 experts of 2048 x 1536 and a shared one: from four tokens on more items than a CTA has warps, and several pieces to each."""
    t = torch()
    L = LargeLayer(2048, 1536, 32, 1, 4, dtype, group, zeros, T, seed=80)
    x = t.randn(T, 2048, generator=t.Generator(device="cuda").manual_seed(T), device="cuda").to(tt(dtype))
    got = L.run(x)
    L.check(x, *got)
    assert all(t.equal(a, b) for a, b in zip(got, L.run(x)))
    assert D.exo_decode_check() == B.OK


@pytest.mark.parametrize("K,alpha", [(256, 0.0), (0, 1.0)])
def test_gemv_without_products_does_not_look_at_the_address_of_x(K, alpha):
    t = torch()
    m = Matrix(70, 256, 64, D.BF16, False, seed=1)
    y = t.full((3, 70), 1.5, device="cuda")
    q = D.Q4(70, K, 64, D.BF16, m.codes.data_ptr(), m.scales.data_ptr())
    q.gemv(3, y.data_ptr() + 1, max(K, 1), y.data_ptr(), 70, D.FP32, alpha, 2.0, stream())
    assert (y == 3).all()
