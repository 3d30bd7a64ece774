"""The feed-forward half of a decoder block on int8 codes: trained straight through the quantizers, then run for single tokens and with experts.

    python examples/int8_feed_forward.py
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1609_07061_amd as q  # noqa: E402

EPS = 1e-5


def codes_of_rows(w):
    """Weights as int8 codes with a scale for every output channel, laid out once per change of the weights.  A channel of zeros has scale 0, one with a value that
    is not finite scale NaN, both codes 0."""
    scale = w.abs().amax(dim=-1).float() / 127
    fine = torch.isfinite(scale) & (scale > 0)
    codes = (w / torch.where(fine, scale, 1.0)[..., None]).round_()
    return torch.where(fine[..., None], codes, 0.0).to(torch.int8), torch.where(torch.isfinite(scale), scale, math.nan)


class FeedForward:
    """h = x + residual; h + down(silu(gate(norm(h))) * up(norm(h))).  Master weights fp32, activations bf16, products on codes."""

    def __init__(self, width, inner, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        init = lambda n, k: torch.randn(n, k, device="cuda", generator=g) / math.sqrt(k)
        self.gamma, self.w1, self.w2 = torch.ones(width, device="cuda"), init(2 * inner, width), init(width, inner)
        self.inner = inner
        self.lay_out()

    def lay_out(self):
        self.codes1, self.codes2 = codes_of_rows(self.w1), codes_of_rows(self.w2)

    def forward(self, x, residual=None):
        a, sa, h = q.qnn_rms_norm_quant(x, self.gamma, EPS, residual)
        u = q.qnn_int8_gemm(a, sa, *self.codes1)
        b, sb = q.qnn_silu_gate_quant(u[:, : self.inner], u[:, self.inner :])
        y = q.qnn_int8_gemm(b, sb, *self.codes2)
        return y, h, (a, sa, h, u, b, sb)

    def backward(self, grad, kept):
        """grad: at h + y -> gradients of h, gamma, w1, w2.  Quantizers count as the identity."""
        a, sa, h, u, b, sb = kept
        values = lambda codes, scale: codes.bfloat16() * scale.bfloat16()[:, None]
        grad_w2 = grad.t() @ values(b, sb)
        grad_b = grad @ values(*self.codes2)
        grad_u = torch.empty_like(u)
        q.qnn_silu_gate_backward(grad_b, u[:, : self.inner], u[:, self.inner :], grad_u[:, : self.inner], grad_u[:, self.inner :])
        grad_w1 = grad_u.t() @ values(a, sa)
        grad_a = grad_u @ values(*self.codes1)
        grad_h, grad_gamma = q.qnn_rms_norm_backward(grad_a, h, self.gamma, EPS, grad_sum=grad)
        return grad_h, grad_gamma, grad_w1, grad_w2

    def step(self, grads, rate):
        for w, g in zip((self.gamma, self.w1, self.w2), grads):
            w -= rate * g.float()
        self.lay_out()


def train(width=256, inner=640, rows=512, steps=60, rate=0.2):
    """Fits one feed-forward part to another one -> the mean square errors step by step."""
    teacher, student = FeedForward(width, inner, 1), FeedForward(width, inner, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, width, device="cuda", generator=g).bfloat16()
    residual = torch.randn(rows, width, device="cuda", generator=g).bfloat16()
    want = teacher.forward(x, residual)[0].float()
    errors = []
    for _ in range(steps):
        y, _, kept = student.forward(x, residual)
        miss = y.float() - want
        errors.append(float(miss.square().mean()))
        grads = student.backward((miss / rows).bfloat16(), kept)
        student.step(grads[1:], rate)
    return errors


class Experts:
    """Norm, router and the chosen experts of a few tokens; every buffer is allocated once, as a server would."""

    def __init__(self, width, inner, experts, top, tokens, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        init = lambda *s: torch.randn(*s, device="cuda", generator=g) / math.sqrt(s[-1])
        self.gamma, self.top = torch.ones(width, device="cuda").bfloat16(), top
        self.router = codes_of_rows(init(experts, width))
        self.first, self.second = codes_of_rows(init(experts, 2 * inner, width)), codes_of_rows(init(experts, width, inner))
        new = lambda *s, dtype: torch.empty(*s, dtype=dtype, device="cuda")
        self.codes, self.scale = new(tokens, width, dtype=torch.int8), new(tokens, dtype=torch.float32)
        self.h, self.out = new(tokens, width, dtype=torch.bfloat16), new(tokens, width, dtype=torch.bfloat16)
        self.logits = new(tokens, experts, dtype=torch.float32)
        self.workspace = new(q.qnn_int8_moe_workspace_bytes(tokens, top, inner), dtype=torch.uint8)

    def forward(self, x, residual):
        q.qnn_rms_norm_quant(x, self.gamma, EPS, residual, self.codes, self.scale, self.h)
        q.qnn_int8_gemm(self.codes, self.scale, *self.router, out=self.logits)
        return q.qnn_int8_moe(self.codes, self.scale, self.logits, self.top, *self.first, *self.second, out=self.out, workspace=self.workspace)


def serve(tokens, width=1024, inner=512, experts=8, top=2, calls=100):
    """The layer with experts as a graph, replayed on new tokens -> (outputs, what the same calls gave outside the graph, us a call)."""
    layer = Experts(width, inner, experts, top, tokens)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, residual = (torch.randn(tokens, width, device="cuda", generator=g).bfloat16() for _ in range(2))
    layer.forward(x, residual)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, residual)
    x.copy_(torch.randn(tokens, width, device="cuda", generator=g))
    want = layer.forward(x, residual).clone()
    layer.out.zero_()
    for _ in range(10):
        graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(calls):
        graph.replay()
    end.record()
    end.synchronize()
    return layer.out, want, begin.elapsed_time(end) * 1e3 / calls


def main():
    errors = train()
    print(f"training: mean square error {errors[0]:.3f} -> {errors[-1]:.3f} in {len(errors)} steps")
    layer = FeedForward(1024, 2816)
    y, h, _ = layer.forward(torch.randn(1, 1024, device="cuda").bfloat16())
    print("one token:", tuple(y.shape), y.dtype)
    for tokens in (1, 16):
        out, want, us = serve(tokens)
        print(f"experts, {tokens} token(s): {us:.1f} us a call as a graph, {'same' if torch.equal(out, want) else 'DIFFERENT'} as outside of it")


if __name__ == "__main__":
    main()
