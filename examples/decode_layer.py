"""One decode step of a layer with 4-bit weights, next to the same layer on a prompt.

The weights of a projection and of a mixture-of-experts layer are quantised on the GPU (exo_q4_quantize).  A few tokens then go
through the projection (exo_gemv_q4_run) and the experts (exo_moe_run) straight from the 4-bit weights; a prompt takes the
projection's weights back to 16 bits (exo_q4_dequantize) and uses the GEMM (exo_gemm_run).  The tokens are the
prompt's last ones, so both ways have to agree.

    python examples/decode_layer.py [--tokens 4] [--hidden 2048] [--inner 1024] [--experts 32] [--top-k 4]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_16389_b200 import binding as B, decode as D  # noqa: E402


class Q4Weights:
    """4-bit weights with their memory: the values of a bf16 matrix, quantised in groups of `group` along k."""

    def __init__(self, w, group=128, zeros=False):
        rows, K = w.shape
        groups = D.padded_k(K) // group
        self.codes = torch.empty(rows, D.padded_k(K) // 2, dtype=torch.uint8, device=w.device)
        self.scales = torch.empty(rows, groups, dtype=torch.bfloat16, device=w.device)
        self.zeros = torch.empty(rows, groups, dtype=torch.uint8, device=w.device) if zeros else None
        self.q = D.Q4(rows, K, group, D.BF16, self.codes.data_ptr(), self.scales.data_ptr(), self.zeros.data_ptr() if zeros else 0)
        self.q.quantize(w.data_ptr(), K, D.BF16, torch.cuda.current_stream().cuda_stream)

    def expert_matrix(self, expert_rows):
        return D.MoeMatrix(self.codes.data_ptr(), 0, expert_rows, self.scales.data_ptr(), 0 if self.zeros is None else self.zeros.data_ptr())


def run(tokens=4, hidden=2048, inner=1024, experts=32, top_k=4, prompt=256, seed=0):
    """(projection of the tokens from 4 bits, the same rows by way of the prompt, the layer's output, taken experts)"""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def weights(rows, K):
        return torch.empty(rows, K, device="cuda", dtype=torch.bfloat16).normal_(0.0, K ** -0.5, generator=gen)

    stream = torch.cuda.current_stream().cuda_stream
    proj = Q4Weights(weights(hidden, hidden))
    gate, up, down = (Q4Weights(weights(experts * r, K)) for r, K in ((inner, hidden), (inner, hidden), (hidden, inner)))
    router = weights(experts, hidden)
    x = torch.empty(prompt, hidden, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)

    # the prompt: 16-bit weights and the GEMM, C = X * W^T (W row-major N x K is a column-major K x N operand)
    w16 = torch.empty(hidden, hidden, device="cuda", dtype=torch.bfloat16)
    proj.q.dequantize(w16.data_ptr(), hidden, D.BF16, stream)
    by_prompt = torch.empty(prompt, hidden, device="cuda", dtype=torch.bfloat16)
    with B.Plan(B.make_desc(prompt, hidden, hidden, B.BF16, B.BF16, B.ROW_MAJOR, B.COL_MAJOR, B.ROW_MAJOR)) as gemm:
        gemm.run(x.data_ptr(), w16.data_ptr(), by_prompt.data_ptr(), stream=stream)
        torch.cuda.synchronize()
        gemm.check()

    # the last tokens: straight from 4 bits, then the experts
    last = x[prompt - tokens:]
    h = torch.empty(tokens, hidden, device="cuda", dtype=torch.bfloat16)
    proj.q.gemv(tokens, last.data_ptr(), hidden, h.data_ptr(), hidden, D.BF16, stream=stream)
    y = torch.empty_like(h)
    taken = torch.empty(tokens, top_k, device="cuda", dtype=torch.int32)
    layer = D.MoeWeights(router.data_ptr(), hidden, gate.expert_matrix(inner), up.expert_matrix(inner), down.expert_matrix(hidden))
    with D.MoePlan(D.MoeDesc(hidden, inner, experts, 0, top_k, tokens, D.BF16, q4_group=128)) as moe:
        moe.run(layer, tokens, h.data_ptr(), hidden, y.data_ptr(), hidden, taken.data_ptr(), stream=stream)
        torch.cuda.synchronize()
    if D.exo_decode_check() != D.OK:
        raise RuntimeError("a device-side wait gave up")
    return h, by_prompt[prompt - tokens:], y, taken


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4), ("hidden", 2048), ("inner", 1024), ("experts", 32), ("top-k", 4)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    h, by_prompt, y, taken = run(a.tokens, a.hidden, a.inner, a.experts, a.top_k)
    off = (h.float() - by_prompt.float()).norm() / by_prompt.float().norm()
    print(f"projection from 4 bits against the prompt's GEMM: relative difference {off:.1e}")
    print(f"experts taken by the first token: {taken[0].tolist()}; layer output of norm {y.float().norm():.4f}")


if __name__ == "__main__":
    main()
