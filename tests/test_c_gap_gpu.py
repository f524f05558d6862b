"""Nothing but the M x N values of C is written, wherever the rows of C end: a TMA store moves pieces of 16 bytes, so a row that ends inside
such a piece and is followed by a gap (ldc beyond the extent) needs its last values stored another way.  Every kernel and every way of
finishing a tile, against the CPU oracle; the gaps and what lies in front of and behind C keep their bits, and C has no room behind its last row.

Tolerance: max |C - Cref| / (sum_k |a b| + |beta c|) <= 1e-3, widened by half an ulp of a 16-bit output type as in the main parity file.
"""
import numpy as np
import pytest

import oracle
from paper_2609_16389_b200 import binding as B
from paper_2609_16389_b200 import harness, synth
from paper_2609_16389_b200.synth import BF16, FP16, FP32

pytestmark = pytest.mark.gpu
TOL = 1e-3
LEAN, PERSISTENT = B.FLAG2_LEAN_ALWAYS, B.FLAG2_LEAN_NEVER | B.FLAG2_SHARE_NEVER
TALL = B.flag2_cta_rows(256) | B.FLAG2_LEAN_NEVER | B.FLAG2_SHARE_NEVER
CANARY, FRONT, BEHIND = 0xA5, 256, 256


def tile(g, bn, extra=0):
    return B.flag_cta_group(g) | B.flag_tile_n(bn) | extra


def problem(M, N, K, ab, cd, la, lb, lc, alpha, beta, more):
    """ldc: the extent rounded up to 16 bytes, and `more` such pieces on top."""
    per = 4 if cd == FP32 else 8
    extent = N if lc == 0 else M
    eight = lambda n: -(-max(n, 1) // 8) * 8  # noqa: E731
    p = synth.Problem("gap", M, N, K, ab, cd, la, lb, lc, alpha, beta, seed=M + 3 * N + 7 * K, dist="normal" if ab == FP16 else "uniform",
                      lda=eight(K if la == 0 else M), ldb=eight(N if lb == 0 else K), ldc=(-(-extent // per) + more) * per)
    assert extent % per, "a row that ends inside a piece"
    return p.generate()


def rows_and_extent(p):
    return (p.M, p.N) if p.c_layout == 0 else (p.N, p.M)


def placed(p, count=1, stride=0):
    """Device bytes: canaries, `count` matrices C without their last row's gap, canaries; and which bytes belong to C."""
    import torch
    cb = 4 if p.c_dtype == FP32 else 2
    rows, extent = rows_and_extent(p)
    size = (rows - 1) * p.ldc * cb + extent * cb
    host = np.full(FRONT + (count - 1) * stride * cb + size + BEHIND, CANARY, np.uint8)
    ours = np.zeros(host.size, bool)
    values = p.C.view(np.uint8).reshape(-1)
    for i in range(count):
        for r in range(rows):
            at, to = r * p.ldc * cb, FRONT + i * stride * cb + r * p.ldc * cb
            host[to:to + extent * cb] = values[at:at + extent * cb]
            ours[to:to + extent * cb] = True
    return torch.from_numpy(host).cuda(), ours


def check(p, dC, ours, at=FRONT, probs=None, info=None):
    out = dC.cpu().numpy()
    assert (out[~ours] == CANARY).all(), ("bytes outside C were written", np.flatnonzero((out != CANARY) & ~ours)[:8], info)
    cb = 4 if p.c_dtype == FP32 else 2
    rows, extent = rows_and_extent(p)
    flat = np.zeros(p.C.size * cb, np.uint8)
    n = (rows - 1) * p.ldc * cb + extent * cb
    flat[:n] = out[at:at + n]
    got = oracle.logical_view(flat.view(synth.storage_np_dtype(p.c_dtype)), p.M, p.N, p.c_layout, p.ldc, p.c_dtype)
    cref, den = oracle.gemm_problem(p)
    gate = TOL * den + oracle.output_rounding_slack(cref, p.c_dtype)
    bad = ~(np.abs(got - cref) <= gate)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5], info)


# M, N, K, ab, cd, la, lb, lc, alpha, beta, pieces of gap beyond the row's last, flags, flags2
CASES = {
    # one tile per CTA: whole and last chunks, a chunk of nothing but the row's end, rows shorter than a piece
    "lean": (300, 201, 136, BF16, BF16, 0, 1, 0, 1.0, 0.0, 0, 0, LEAN),
    "lean_beta": (300, 201, 136, FP16, FP16, 0, 1, 0, 1.5, -0.5, 1, 0, LEAN),
    "lean_fp32": (140, 99, 72, BF16, FP32, 0, 1, 0, 1.0, 0.75, 0, 0, LEAN),
    "lean_end_alone": (140, 67, 72, BF16, BF16, 0, 1, 0, 1.0, 0.5, 2, 0, LEAN),
    "lean_end_alone_fp32": (140, 33, 72, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, 0, LEAN),
    "lean_short_rows": (70, 3, 72, BF16, BF16, 0, 1, 0, 1.0, 1.0, 1, 0, LEAN),
    "lean_one_value": (1, 1, 8, BF16, FP32, 0, 1, 0, 2.0, 0.0, 1, 0, LEAN),
    "lean_wide": (257, 205, 520, BF16, BF16, 0, 1, 0, 1.0, 1.0, 0, B.flag_tile_n(128), LEAN),
    "lean_two": (140, 131, 2048, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, B.flag_split_k(2), LEAN),
    "lean_four": (140, 131, 4096, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, B.flag_split_k(4), LEAN),
    "lean_pair": (600, 333, 200, BF16, BF16, 0, 1, 0, 1.0, 0.0, 1, tile(2, 256), LEAN),
    "lean_pair_beta": (600, 131, 200, FP16, FP32, 0, 1, 0, -1.0, 0.5, 0, tile(2, 128), LEAN),
    # the persistent kernel's tile shapes, with one and two staging buffers
    "p1x64": (300, 131, 136, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, tile(1, 64), PERSISTENT),
    "p1x128": (300, 259, 136, BF16, FP32, 0, 1, 0, 1.0, 0.5, 0, tile(1, 128, B.flag_epi_buffers(2)), PERSISTENT),
    "p1x256": (300, 515, 136, FP16, FP16, 0, 1, 0, 1.0, 0.0, 0, tile(1, 256), PERSISTENT),
    "p2x128": (600, 387, 136, BF16, BF16, 1, 0, 0, 1.0, 1.0, 1, tile(2, 128, B.flag_epi_buffers(2)), PERSISTENT),
    "p2x256": (600, 515, 264, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, tile(2, 256), PERSISTENT),
    "p2x256_end_alone": (600, 321, 264, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, tile(2, 256, B.flag_epi_buffers(1)), PERSISTENT),
    "short_rows": (600, 5, 264, BF16, BF16, 0, 1, 0, 1.0, 0.0, 0, tile(2, 256), PERSISTENT),
    "many_tiles": (2100, 1027, 200, BF16, BF16, 0, 1, 0, 1.0, 0.0, 0, tile(2, 128, B.flag_grid_limit(8)), PERSISTENT),
    "columns": (203, 300, 136, BF16, BF16, 0, 1, 1, 1.0, 0.5, 0, 0, 0),
    "columns_fp32": (515, 600, 136, FP16, FP32, 1, 0, 1, 1.0, 0.0, 0, tile(2, 256), PERSISTENT),
    "tf32": (300, 203, 132, FP32, FP32, 0, 1, 0, 1.0, 0.5, 0, 0, 0),
    "tall": (1100, 515, 200, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, tile(2, 256), TALL),
    "tall_fp32": (1100, 515, 200, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, tile(2, 256), TALL),
    "shared": (520, 1027, 264, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, 0, B.FLAG2_SHARE_ALWAYS),
    "substituted": (520, 1027, 264, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, 0, B.FLAG2_SHARE_SUBSTITUTED),
    # tiles whose K is cut: the owner adds, or finds its accumulator filled; parts that are added onto C
    "cut": (640, 521, 4096, BF16, FP32, 0, 1, 0, 0.75, 0.5, 0, tile(2, 256, B.flag_split_k(4)), PERSISTENT),
    "cut_16_bit": (640, 521, 4096, BF16, BF16, 0, 1, 0, 0.75, 0.0, 0, tile(1, 128, B.flag_split_k(4)), PERSISTENT),
    "cut_behind_waves": (1300, 521, 2048, BF16, BF16, 0, 1, 0, 1.0, 0.0, 0, tile(1, 128, B.flag_split_k(3) | B.flag_grid_limit(20)), PERSISTENT),
    "added": (640, 521, 4096, BF16, FP32, 0, 1, 0, 0.75, 0.0, 0, tile(2, 256, B.FLAG_SPLIT_REDUCE_ADD | B.flag_split_k(4)), PERSISTENT),
    "added_onto": (640, 521, 4096, BF16, FP32, 0, 1, 0, 0.75, 1.0, 0, tile(1, 128, B.FLAG_SPLIT_REDUCE_ADD | B.flag_split_k(4)), PERSISTENT),
    # nothing is multiplied
    "no_depth": (300, 201, 0, BF16, BF16, 0, 1, 0, 1.0, 0.5, 0, 0, 0),
    "alpha_zero": (300, 201, 136, BF16, FP32, 0, 1, 0, 0.0, 0.5, 0, tile(2, 128), PERSISTENT),
    # results beyond L2 (stores with a priority)
    "large": (4100, 4099, 64, BF16, FP32, 0, 1, 0, 1.0, 0.0, 0, 0, 0),
}


@pytest.mark.parametrize("name", CASES)
def test_only_c_is_written(name):
    import torch
    M, N, K, ab, cd, la, lb, lc, alpha, beta, more, flags, flags2 = CASES[name]
    if flags2 & 3 >= 2 and not B.exo_gemm_has_shared_operand_clusters():
        pytest.skip("this deployment carries the base library only")
    p = problem(M, N, K, ab, cd, la, lb, lc, alpha, beta, more)
    dA, dB = harness._to_device(p.A, "cuda:0"), harness._to_device(p.B, "cuda:0")
    dC, ours = placed(p)
    with B.Plan(harness.desc_of(p, flags, flags2=flags2)) as plan:
        info = plan.info()
        plan.run(dA.data_ptr(), dB.data_ptr(), dC.data_ptr() + FRONT, alpha, beta, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        plan.check()
    check(p, dC, ours, info=info)


@pytest.mark.parametrize("cd,beta,lc,flags", [(BF16, 0.5, 0, 0), (FP32, 0.0, 0, 0), (BF16, 0.0, 1, tile(1, 128)), (FP32, 1.0, 0, tile(2, 256))])
def test_only_the_matrices_of_a_batch_are_written(cd, beta, lc, flags):
    import torch
    count = 3
    p = problem(131, 203, 136, BF16, cd, 0, 1, lc, 1.0, beta, 0)
    dA, dB = harness._to_device(np.tile(p.A, count), "cuda:0"), harness._to_device(np.tile(p.B, count), "cuda:0")
    stride = p.C.size + 16
    dC, ours = placed(p, count, stride)
    with B.Plan(harness.desc_of(p, flags), batch=(count, p.A.size, p.B.size, stride)) as plan:
        plan.run(dA.data_ptr(), dB.data_ptr(), dC.data_ptr() + FRONT, p.alpha, beta, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        plan.check()
    for i in range(count):
        check(p, dC, ours, FRONT + i * stride * (4 if cd == FP32 else 2))


@pytest.mark.parametrize("case", ["lean_beta", "p2x256", "columns", "short_rows"])
def test_only_c_is_written_without_a_plan(case):
    import torch
    M, N, K, ab, cd, la, lb, lc, alpha, beta, more, flags, flags2 = CASES[case]
    p = problem(M, N, K, ab, cd, la, lb, lc, alpha, beta, more)
    dA, dB = harness._to_device(p.A, "cuda:0"), harness._to_device(p.B, "cuda:0")
    dC, ours = placed(p)
    st, detail = B.exo_gemm_run_static(harness.desc_of(p, flags, flags2=flags2), dA.data_ptr(), dB.data_ptr(), dC.data_ptr() + FRONT, alpha, beta,
                                       torch.cuda.current_stream().cuda_stream, blocking=True)
    assert st == B.OK, detail
    check(p, dC, ours)


def test_neighbouring_column_slices():
    """Column slices of one matrix, each written by a product of its own, in either order: neither touches the other's."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    M, K = 300, 136   # the second slice starts on 16 bytes, the first ends inside a piece
    a = torch.randn(M, K, device="cuda", generator=g).bfloat16()
    c = torch.zeros(M, 416, device="cuda", dtype=torch.bfloat16)
    parts = []
    for lo, hi in ((0, 205), (208, 411)):
        b = torch.randn(hi - lo, K, device="cuda", generator=g).bfloat16()
        parts.append((lo, hi, b, B.Plan(B.make_desc(M, hi - lo, K, BF16, BF16, 0, 1, 0, lda=K, ldb=K, ldc=416))))
    for order in (parts, parts[::-1]):
        c.fill_(3.0)
        for lo, hi, b, plan in order:
            plan.run(a.data_ptr(), b.data_ptr(), c.data_ptr() + 2 * lo, 1.0, 0.0, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for lo, hi, b, plan in order:
            plan.check()
            want = a.double() @ b.double().t()
            # the sum in fp32 (K * 2^-23 of the magnitudes' sum), then half a step of bf16
            bound = K * 2.0 ** -23 * (a.double().abs() @ b.double().abs().t())
            assert ((c[:, lo:hi].double() - want).abs() <= bound + 2.0 ** -8 * (want.abs() + bound)).all()
        assert (c[:, 205:208] == 3.0).all() and (c[:, 411:] == 3.0).all()
