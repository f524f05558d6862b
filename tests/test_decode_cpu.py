"""The few-token operators' C ABI on the host: exports, argument checks, the 4-bit layout."""
import os
import re

import numpy as np
import pytest

from paper_2609_16389_b200 import binding as B
from paper_2609_16389_b200 import decode as D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # a non-null, aligned address that no refused call reads


def test_library_exports_every_symbol_of_the_header():
    text = open(os.path.join(ROOT, "include", "exo_decode.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(exo_\w+)\s*\(", text))
    assert declared == set(D.EXPORTED_SYMBOLS)
    for name in declared:
        assert hasattr(D.lib(), name)


def q4(rows=64, K=256, group=128, dtype=D.BF16, codes=P, scales=P, zeros=0):
    return D.Q4Struct(rows, K, group, dtype, codes, scales, zeros)


@pytest.mark.parametrize("call", [D.exo_q4_quantize, D.exo_q4_dequantize])
def test_quantisation_refuses_bad_arguments(call):
    assert call(None, P, 256, D.BF16) == B.ERR_NULL
    assert call(q4(), 0, 256, D.BF16) == B.ERR_NULL
    assert call(q4(codes=0), P, 256, D.BF16) == B.ERR_NULL
    assert call(q4(scales=0), P, 256, D.BF16) == B.ERR_NULL
    assert call(q4(rows=-1), P, 256, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(K=-1), P, 256, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(K=(1 << 30) + 1), P, 1 << 31, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(group=16), P, 256, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(dtype=D.FP32), P, 256, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(), P, 255, D.BF16) == B.ERR_INVALID_ARG
    assert call(q4(), P, 256, 3) == B.ERR_INVALID_ARG
    assert call(q4(codes=P + 8), P, 256, D.BF16) == B.ERR_ALIGNMENT
    assert call(q4(scales=P + 1), P, 256, D.BF16) == B.ERR_ALIGNMENT
    assert call(q4(scales=P + 4, group=32), P, 256, D.BF16) == B.ERR_ALIGNMENT
    assert call(q4(zeros=P + 1, group=64), P, 256, D.BF16) == B.ERR_ALIGNMENT
    assert call(q4(), P + 1, 256, D.BF16) == B.ERR_ALIGNMENT
    assert call(q4(), P + 2, 256, D.FP32) == B.ERR_ALIGNMENT
    assert call(q4(rows=0, codes=0, scales=0), 0, 256, D.BF16) == B.OK
    assert call(q4(K=0, codes=0, scales=0), 0, 1, D.BF16) == B.OK


def test_gemv_refuses_bad_arguments():
    run = D.exo_gemv_q4_run
    assert run(None, 1, P, 256, P, 64, D.BF16) == B.ERR_NULL
    assert run(q4(), 1, 0, 256, P, 64, D.BF16) == B.ERR_NULL
    assert run(q4(), 1, P, 256, 0, 64, D.BF16) == B.ERR_NULL
    assert run(q4(codes=0), 1, P, 256, P, 64, D.BF16) == B.ERR_NULL
    assert run(q4(), -1, P, 256, P, 64, D.BF16) == B.ERR_INVALID_ARG
    assert run(q4(), 1, P, 255, P, 64, D.BF16) == B.ERR_INVALID_ARG
    assert run(q4(), 1, P, 256, P, 63, D.BF16) == B.ERR_INVALID_ARG
    assert run(q4(), 1, P, 256, P, 64, D.FP16) == B.ERR_INVALID_ARG      # neither fp32 nor W's type
    assert run(q4(group=48), 1, P, 256, P, 64, D.BF16) == B.ERR_INVALID_ARG
    assert run(q4(), 65, P, 256, P, 64, D.BF16) == B.ERR_UNSUPPORTED
    assert run(q4(codes=P + 4), 1, P, 256, P, 64, D.BF16) == B.ERR_ALIGNMENT
    assert run(q4(), 1, P + 1, 256, P, 64, D.BF16) == B.ERR_ALIGNMENT
    assert run(q4(), 1, P, 256, P + 2, 64, D.FP32) == B.ERR_ALIGNMENT
    assert run(q4(), 0, 0, 256, 0, 64, D.BF16) == B.OK
    assert run(q4(rows=0), 1, 0, 256, 0, 64, D.BF16) == B.OK


def desc(**kw):
    return D.MoeDesc(**{**dict(hidden=64, inner=32, experts=4, shared=0, top_k=2, max_tokens=8, dtype=D.BF16), **kw})


def test_moe_validate():
    assert D.exo_moe_validate(desc()) == B.OK
    assert D.exo_moe_validate(desc(hidden=1, inner=1, experts=1, top_k=1, max_tokens=1)) == B.OK
    assert D.exo_moe_validate(desc(experts=512, shared=8, top_k=16, max_tokens=64, q4_group=32, dtype=D.FP16)) == B.OK
    assert D.exo_moe_validate(None) == B.ERR_NULL
    for bad in (dict(hidden=0), dict(inner=0), dict(hidden=1 << 25), dict(inner=1 << 25), dict(experts=0), dict(shared=-1),
                dict(top_k=0), dict(top_k=5), dict(max_tokens=0), dict(dtype=D.FP32), dict(q4_group=16), dict(renormalize=2),
                dict(device=-2)):
        assert D.exo_moe_validate(desc(**bad)) == B.ERR_INVALID_ARG, bad
    for big in (dict(experts=513), dict(shared=9), dict(experts=32, top_k=17), dict(max_tokens=65)):
        assert D.exo_moe_validate(desc(**big)) == B.ERR_UNSUPPORTED, big


def test_moe_entry_points_take_null():
    assert D.exo_moe_destroy(None) == B.OK
    assert D.exo_moe_workspace_bytes(None) == 0
    assert D.exo_moe_run(None, None, 1, P, 64, P, 64) == B.ERR_NULL
    assert D.lib().exo_moe_create(None, desc()) == B.ERR_NULL
    st, h = D.exo_moe_create(desc(top_k=9))
    assert st == B.ERR_INVALID_ARG and h is None


@pytest.mark.parametrize("rows,K", [(1, 1), (3, 127), (2, 128), (5, 300), (1, 512)])
def test_pack_codes_follows_the_layout(rows, K):
    codes = np.random.default_rng(K).integers(0, 16, (rows, K), dtype=np.uint8)
    words = D.pack_codes(codes).view("<u4")
    assert words.shape == (rows, D.padded_k(K) // 8)
    for r in range(rows):
        for k in range(K):
            b, j, t, i = k // 128, k % 128 // 32, k % 32 // 8, k % 8
            n = i // 2 + 4 * (i % 2)
            assert (int(words[r, 16 * b + 4 * t + j]) >> 4 * n) & 15 == codes[r, k]


def test_debug_set_refuses_bad_arguments():
    for bad in ((-1, 0), (10001, 0), (20, -1), (20, 3)):
        assert D.exo_decode_debug_set(*bad) == B.ERR_INVALID_ARG
    assert D.exo_decode_debug_set(20, 2) == B.OK and D.exo_decode_debug_set(0, 0) == B.OK
