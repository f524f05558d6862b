"""What exo_fused.h refuses, and the 64-bit references of its GPU tests, without a GPU."""
import ctypes
import math
import os
import re

import pytest
import torch

import fused_reference as R
from paper_2609_16389_b200 import binding as B
from paper_2609_16389_b200 import fused as E

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 2, 3, 4


def test_symbols_and_structs():
    text = open(os.path.join(ROOT, "include", "exo_fused.h")).read()
    declared = set(re.findall(r"\b(exo_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert declared == set(E.EXPORTED_SYMBOLS)
    for name in declared:
        assert hasattr(B.lib(), name), name
    # the C layouts: eight-byte fields first in each run, four-byte ones packed between them
    assert ctypes.sizeof(E.FfnDesc) == 3 * 8 + 4 * 4 + 4 * 8 + 8
    assert ctypes.sizeof(E.CeDesc) == 3 * 8 + 4 * 4 + 5 * 8 + 8
    assert ctypes.sizeof(E.I8Struct) == 5 * 8
    assert E.CeDesc.ignore_index.offset == 40 and E.FfnDesc.ldx.offset == 40


def ffn(**kw):
    args = dict(tokens=4, hidden=64, inner=96, dtype=E.BF16)
    args.update(kw)
    return E.FfnDesc(**args)


@pytest.mark.parametrize("kw,status", [
    ({}, OK), (dict(tokens=0), OK), (dict(hidden=1, inner=1), OK), (dict(ldx=65, ldy=64, ld_gate_up=71, ld_down=96), OK),
    (dict(dtype=E.FP16, activation=E.GELU_TANH, training=1, grad_dtype=E.FP16), OK), (dict(training=1, grad_dtype=E.FP32), OK),
    (dict(tokens=-1), INVALID), (dict(hidden=0), INVALID), (dict(inner=0), INVALID), (dict(tokens=(1 << 24) + 1), INVALID),
    (dict(dtype=E.FP32), INVALID), (dict(dtype=7), INVALID), (dict(activation=3), INVALID), (dict(activation=-1), INVALID),
    (dict(training=2), INVALID), (dict(training=1, grad_dtype=E.FP16), INVALID), (dict(grad_dtype=9), OK),   # not read without training
    (dict(training=1, grad_dtype=9), INVALID), (dict(ldx=63), INVALID), (dict(ldy=1), INVALID), (dict(ld_gate_up=63), INVALID),
    (dict(ld_down=95), INVALID), (dict(ld_down=-96), INVALID), (dict(ldx=1 << 40), INVALID), (dict(device=-2), INVALID)])
def test_ffn_descriptors(kw, status):
    assert E.exo_ffn_validate(ffn(**kw)) == status
    if status:
        assert E.exo_ffn_create(ffn(**kw)) == (status, None)


def ce(**kw):
    args = dict(tokens=4, hidden=64, vocab=1000, dtype=E.FP16)
    args.update(kw)
    return E.CeDesc(**args)


@pytest.mark.parametrize("kw,status", [
    ({}, OK), (dict(tokens=0), OK), (dict(vocab=1, hidden=1), OK), (dict(label_smoothing=0.5, ignore_index=-(1 << 63)), OK),
    (dict(training=1, grad_dtype=E.FP16, keep_bytes=0, piece=256), OK), (dict(training=1, grad_dtype=E.FP32, keep_bytes=1 << 40), OK),
    (dict(tokens=-1), INVALID), (dict(hidden=0), INVALID), (dict(vocab=0), INVALID), (dict(vocab=(1 << 24) + 1), INVALID),
    (dict(dtype=E.FP32), INVALID), (dict(training=-1), INVALID), (dict(training=1, grad_dtype=E.BF16), INVALID),
    (dict(label_smoothing=-0.1), INVALID), (dict(label_smoothing=1.0), INVALID), (dict(label_smoothing=math.nan), INVALID),
    (dict(keep_bytes=-2), INVALID), (dict(piece=-1), INVALID), (dict(ldx=63), INVALID), (dict(ldw=-64), INVALID), (dict(device=-5), INVALID)])
def test_ce_descriptors(kw, status):
    assert E.exo_ce_validate(ce(**kw)) == status
    if status:
        assert E.exo_ce_create(ce(**kw)) == (status, None)


def test_null_plans_and_descriptors():
    L = E.lib()
    assert L.exo_ffn_validate(None) == L.exo_ce_validate(None) == NULL
    assert L.exo_ffn_create(None, ffn()) == L.exo_ce_create(None, ce()) == NULL
    assert E.exo_ffn_forward(None, 0, 0, 0, 0) == E.exo_ffn_backward(None, 0, 0, 0, 0, 0) == NULL
    assert E.exo_ce_forward(None, 0, 0, 0) == E.exo_ce_backward(None, 0, 0, 0, 0, 0) == NULL
    assert E.exo_ffn_check(None) == E.exo_ce_check(None) == NULL
    assert E.exo_ffn_saved_bytes(None) == E.exo_ce_saved_bytes(None) == E.exo_ffn_workspace_bytes(None) == E.exo_ce_workspace_bytes(None) == 0
    assert E.exo_ffn_destroy(None) == E.exo_ce_destroy(None) == OK
    assert E.exo_fused_debug_set(-1, 0) == E.exo_fused_debug_set(10001, 0) == E.exo_fused_debug_set(0, 2) == INVALID


def i8(rows=4, K=100, ld=112, codes=256, scales=256):
    return E.I8Struct(rows, K, ld, codes, scales)


@pytest.mark.parametrize("q,x,ldx,dtype,status", [
    (i8(rows=-1), 256, 100, E.BF16, INVALID), (i8(K=-1), 256, 100, E.BF16, INVALID), (i8(ld=96), 256, 100, E.BF16, INVALID),
    (i8(), 256, 99, E.BF16, INVALID), (i8(), 256, 100, 3, INVALID), (i8(), 0, 100, E.BF16, NULL), (i8(codes=0), 256, 100, E.BF16, NULL),
    (i8(scales=0), 256, 100, E.BF16, NULL), (i8(codes=264), 256, 100, E.BF16, ALIGNMENT), (i8(scales=258), 256, 100, E.BF16, ALIGNMENT),
    (i8(ld=104), 256, 100, E.BF16, ALIGNMENT), (i8(), 257, 100, E.FP16, ALIGNMENT), (i8(), 258, 100, E.FP32, ALIGNMENT),
    (i8(rows=0, codes=0, scales=0), 0, 100, E.BF16, OK)])
def test_i8_quantize_refusals(q, x, ldx, dtype, status):
    assert E.exo_i8_quantize(q, x, ldx, dtype) == status


@pytest.mark.parametrize("x,w,y,ldy,dtype,alpha,status", [
    (i8(rows=2), i8(K=99), 256, 4, E.BF16, 1.0, INVALID), (i8(rows=2), i8(), 256, 3, E.BF16, 1.0, INVALID), (i8(), i8(), 256, 4, 5, 1.0, INVALID),
    (i8(ld=16), i8(), 256, 4, E.BF16, 1.0, INVALID), (i8(), i8(), 0, 4, E.BF16, 1.0, NULL), (i8(codes=0), i8(), 256, 4, E.BF16, 1.0, NULL),
    (i8(), i8(scales=0), 256, 4, E.BF16, 1.0, NULL), (i8(codes=8), i8(), 256, 4, E.BF16, 1.0, ALIGNMENT), (i8(), i8(ld=120), 256, 4, E.BF16, 1.0, ALIGNMENT),
    (i8(), i8(), 257, 4, E.BF16, 1.0, ALIGNMENT), (i8(), i8(), 258, 4, E.FP32, 1.0, ALIGNMENT),
    (i8(K=131072, ld=131072), i8(K=131072, ld=131072), 256, 4, E.BF16, 1.0, UNSUPPORTED), (i8(rows=0), i8(), 0, 4, E.BF16, 1.0, OK),
    (i8(), i8(rows=0), 0, 4, E.BF16, 1.0, OK)])
def test_i8_gemm_refusals(x, w, y, ldy, dtype, alpha, status):
    assert E.exo_gemm_i8_run(x, w, y, ldy, dtype, alpha) == status


def test_null_matrices():
    L = E.lib()
    assert L.exo_i8_quantize(None, 256, 100, E.BF16, None) == NULL
    assert L.exo_gemm_i8_run(None, i8(), 256, 4, E.BF16, 1.0, 0.0, None) == L.exo_gemm_i8_run(i8(), None, 256, 4, E.BF16, 1.0, 0.0, None) == NULL


def test_without_a_device_nothing_is_made():
    if torch.cuda.is_available():
        pytest.skip("a device is there")
    for create, desc in ((E.exo_ffn_create, ffn()), (E.exo_ce_create, ce())):
        st, handle = create(desc)
        assert st != OK and handle is None
    assert E.exo_gemm_i8_run(i8(), i8(), 256, 4, E.BF16) != OK


# ---------------------------------------------------------------- the references themselves
def test_reference_gradients():
    """The formulas of the reference against automatic differentiation in 64 bits (their values, not their bounds)."""
    g = torch.Generator().manual_seed(1)
    x, gu, d, dy = (torch.randn(*s, generator=g).bfloat16() for s in ((5, 12), (16, 12), (12, 8), (5, 12)))
    for act in R.ACTS:
        X, GU, D = (t.double().requires_grad_() for t in (x, gu, d))
        y = (R.ACTS[act](X @ GU[:8].t()) * (X @ GU[8:].t())) @ D.t()
        want = torch.autograd.grad(y, (X, GU, D), dy.double())
        got = R.ffn(x, gu, d, act, dy)
        for v, name in zip((y, *want), ("y", "dx", "dgate_up", "ddown")):
            assert torch.allclose(got[name][0], v.detach(), rtol=1e-12, atol=1e-12), (act, name)
    w = torch.randn(30, 12, generator=g).bfloat16()
    target, r = torch.tensor([3, -100, 29, 7, 30]), torch.rand(5, generator=g)
    X, W = x.double().requires_grad_(), w.double().requires_grad_()
    safe = torch.where((target >= 0) & (target < 30), target, -100)
    for s in (0.0, 0.2):
        loss = torch.nn.functional.cross_entropy(X @ W.t(), safe, ignore_index=-100, label_smoothing=s, reduction="none")
        want = torch.autograd.grad((loss * r.double()).sum(), (X, W))
        got = R.ce(x, w, target, s, -100, r)
        assert torch.allclose(got["loss"][0], loss.detach(), rtol=1e-12, atol=1e-12)
        for v, name in zip(want, ("dx", "dw")):
            assert torch.allclose(got[name][0], v, rtol=1e-11, atol=1e-12), name


def test_reference_quantisation_is_fp32_division():
    x = torch.tensor([[1.0, -127.0, 0.5, 63.5], [0.0, 0.0, 0.0, 0.0], [3.0, 1.0, -1.0, 1.5]])
    codes, scales = R.quantized(x)
    assert scales.tolist()[:2] == [1.0, 0.0]
    assert codes.tolist()[0] == [1, -127, 0, 64] and codes.tolist()[1] == [0, 0, 0, 0] and codes.tolist()[2][:1] == [127]
