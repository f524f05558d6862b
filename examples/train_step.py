"""One training step of a feed-forward block under a language model's head, and the trained head in 8 bits.

A residual block y = x + ffn(x) (exo_ffn_forward) is followed by the cross entropy of a head over a vocabulary (exo_ce_forward); the gradients
come back through both (exo_ce_backward, exo_ffn_backward) and the weights take a step.  Neither the logits nor the block's inner gradients
are kept longer than the step.  The head is then quantised (exo_i8_quantize) and scores a few tokens (exo_gemm_i8_run), and the same
quantities from automatic differentiation in fp32 are printed next to it all.

    python examples/train_step.py [--tokens 512] [--hidden 512] [--inner 1408] [--vocab 8003] [--steps 3]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_16389_b200 import fused as E  # noqa: E402


class Step:
    """The plans, the weights and the memory of a step for a fixed number of tokens."""

    def __init__(self, tokens, hidden, inner, vocab, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weights(rows, cols, deviation):
            return torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16).normal_(0.0, deviation, generator=g)

        self.shape = tokens, hidden, inner, vocab
        self.x = weights(tokens, hidden, 1.0)
        self.target = torch.randint(0, vocab, (tokens,), device="cuda", generator=g)
        self.target[::17] = -100                                   # padding
        self.gate_up, self.down, self.head = weights(2 * inner, hidden, hidden ** -0.5), weights(hidden, inner, inner ** -0.5), weights(vocab, hidden, hidden ** -0.5)
        self.block = E.FfnPlan(E.FfnDesc(tokens, hidden, inner, E.BF16, E.SILU, training=1, grad_dtype=E.FP32))
        self.loss_head = E.CePlan(E.CeDesc(tokens, hidden, vocab, E.BF16, training=1, grad_dtype=E.FP32))
        self.saved = torch.empty(self.block.saved_bytes(), device="cuda", dtype=torch.uint8)
        self.saved_head = torch.empty(self.loss_head.saved_bytes(), device="cuda", dtype=torch.uint8)
        self.y, self.h, self.dh, self.dx = (torch.empty_like(self.x) for _ in range(4))
        self.loss, self.lse = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
        self.dloss = (self.target >= 0).float() / (self.target >= 0).sum()   # the mean over the tokens that count
        self.d_gate_up, self.d_down, self.d_head = (torch.empty(w.shape, device="cuda") for w in (self.gate_up, self.down, self.head))

    def forward(self):
        s = torch.cuda.current_stream().cuda_stream
        self.block.forward(self.x.data_ptr(), self.gate_up.data_ptr(), self.down.data_ptr(), self.y.data_ptr(), self.saved.data_ptr(), s)
        torch.add(self.x, self.y, out=self.h)
        self.loss_head.forward(self.h.data_ptr(), self.head.data_ptr(), self.target.data_ptr(), self.loss.data_ptr(), self.lse.data_ptr(),
                               self.saved_head.data_ptr(), s)
        return torch.dot(self.loss, self.dloss)

    def backward(self):
        s = torch.cuda.current_stream().cuda_stream
        self.loss_head.backward(self.h.data_ptr(), self.head.data_ptr(), self.target.data_ptr(), self.lse.data_ptr(), self.dloss.data_ptr(),
                                self.saved_head.data_ptr(), self.dh.data_ptr(), self.d_head.data_ptr(), stream=s)
        self.block.backward(self.x.data_ptr(), self.gate_up.data_ptr(), self.down.data_ptr(), self.saved.data_ptr(), self.dh.data_ptr(),
                            self.dx.data_ptr(), self.d_gate_up.data_ptr(), self.d_down.data_ptr(), stream=s)
        self.dx += self.dh                                         # the residual path

    def update(self, rate):
        for w, d in ((self.gate_up, self.d_gate_up), (self.down, self.d_down), (self.head, self.d_head)):
            w.copy_(w.float() - rate * d)

    def by_autograd(self):
        """(loss, gradients of x, gate_up, down, head) in fp32, from the bf16 weights."""
        inner = self.shape[2]
        x, gu, d, w = (t.float().requires_grad_() for t in (self.x, self.gate_up, self.down, self.head))
        h = x + (torch.nn.functional.silu(x @ gu[:inner].t()) * (x @ gu[inner:].t())) @ d.t()
        loss = torch.nn.functional.cross_entropy(h @ w.t(), self.target, ignore_index=-100)
        return loss.detach(), torch.autograd.grad(loss, (x, gu, d, w))

    def scores_in_8_bits(self, tokens=4):
        """Logits of the first tokens from 8-bit codes, and in fp32."""
        _, hidden, _, vocab = self.shape
        s = torch.cuda.current_stream().cuda_stream
        ld = (hidden + 15) // 16 * 16
        codes = [torch.empty(n, ld, device="cuda", dtype=torch.int8) for n in (tokens, vocab)]
        scales = [torch.empty(n, device="cuda") for n in (tokens, vocab)]
        q = [E.I8(n, hidden, ld, c.data_ptr(), z.data_ptr()) for n, c, z in zip((tokens, vocab), codes, scales)]
        q[0].quantize(self.h.data_ptr(), hidden, E.BF16, s)
        q[1].quantize(self.head.data_ptr(), hidden, E.BF16, s)
        logits = torch.empty(tokens, vocab, device="cuda")
        q[1].gemm(q[0], logits.data_ptr(), vocab, E.FP32, stream=s)
        return logits, self.h[:tokens].float() @ self.head.float().t()


def off(a, b):
    return ((a.float() - b.float()).norm() / b.float().norm()).item()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 512), ("hidden", 512), ("inner", 1408), ("vocab", 8003), ("steps", 3)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    step = Step(a.tokens, a.hidden, a.inner, a.vocab)
    for i in range(a.steps):
        want, grads = step.by_autograd()
        loss = step.forward()
        step.backward()
        far = max(off(x, y) for x, y in zip((step.dx, step.d_gate_up, step.d_down, step.d_head), grads))
        print(f"step {i}: loss {loss.item():.4f} (autograd in fp32: {want.item():.4f}), gradients within {far:.1e}")
        step.update(0.5)
    step.block.check()
    step.loss_head.check()
    got, want = step.scores_in_8_bits()
    print(f"logits of four tokens in 8 bits: relative difference {off(got, want):.1e}")


if __name__ == "__main__":
    main()
