"""A mixture-of-experts block with its experts held in 8-bit floating point, as a program serves it and fine-tunes its router.

    python examples/fp8_experts.py [--tokens 4096] [--d-model 1024] [--d-ff 4096] [--experts 64] [--top-k 2]

Forward, six calls of the library: route, group the rows by expert, quantise the hidden states on their way to the experts, the two
products (the hidden activation goes from one to the other in 8 bits), combine.  Backward, with the quantisation taken as the identity:
the gradient of the hidden states through the transposed weights, rows in e5m2, and that of the router's logits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2308_12066_amd import binding as B  # noqa: E402


def _codes(rows, cols, dtype=torch.float8_e4m3fn):
    blocks = B.fp8_blocks(cols)
    return torch.empty(rows, blocks * B.FP8_BLOCK, dtype=dtype, device="cuda"), torch.empty(blocks, rows, device="cuda")


class Block:
    """w1 [E, d, f], w2 [E, f, d]: quantised here, once, in both orientations.  gate [d, E] float32."""

    def __init__(self, w1, w2, gate, top_k, max_tokens, **router):
        self.E, self.d, self.f = w1.shape
        self.k, self.T, self.gate = top_k, max_tokens, gate
        self.router = B.Router(self.E, top_k, **router)
        self.ctx = B.Context(B.make_config(self.d, 64, self.E, top_k, 1, max_tokens, B.BF16))  # for grouping and combining
        self.w = []
        for w, n_in, n_out in ((w1, self.d, self.f), (w2, self.f, self.d)):
            both = []
            for a, b in ((n_in, n_out), (n_out, n_in)):
                q, s = B.fp8_weight_shapes(self.E, a, b)
                both += [torch.empty(q, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(s, device="cuda")]
            B.quantize_weights(w.contiguous(), *both)
            self.w.append(both)
        R = max_tokens * top_k
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        self.idx, self.weight = new(max_tokens, top_k, dtype=torch.int32), new(max_tokens, top_k, dtype=torch.float32)
        self.row_of, self.offsets = new(R, dtype=torch.int32), new(self.E + 1, dtype=torch.int32)
        self.x_q, self.h_q, self.y_rows = _codes(R, self.d), _codes(R, self.f), new(R, self.d)
        self.y = new(max_tokens, self.d)

    def close(self):
        torch.cuda.synchronize()
        self.ctx.close()

    def logits(self, x):
        return x.float() @ self.gate

    def forward(self, x, logits, stream=None):
        """x [T, d] bf16, logits [T, E] -> y [T, d] bf16 (this block's buffer), on `stream` or torch's current one.  Nothing is allocated:
        it may be captured into a graph."""
        stream = stream or torch.cuda.current_stream()   # a context's calls take the null stream otherwise
        (w1, s1), (w2, s2) = self.w[0][:2], self.w[1][:2]
        self.router.route(logits, None, self.idx, self.weight, None, stream)
        self.ctx.group_rows(self.idx, self.T, self.row_of, self.offsets, stream)
        B.quantize_rows(x, *self.x_q, self.row_of, self.k, stream)
        B.expert_matmul(*self.x_q, w1, s1, self.offsets, self.d, self.f, *self.h_q, relu=True, stream=stream)
        B.expert_matmul(*self.h_q, w2, s2, self.offsets, self.f, self.d, self.y_rows, stream=stream)
        self.ctx.combine(self.y_rows, self.row_of, self.weight, self.T, self.y, stream=stream)
        return self.y

    def backward(self, logits, d_y, stream=None):
        """d_y [T, d] float32, after forward() on the same logits -> (d_x through the experts [T, d] bf16, d_logits [T, E]), on `stream` or
        torch's current one, like forward(): torch's operations and the library's one behind the other."""
        stream = stream or torch.cuda.current_stream()
        with torch.cuda.stream(stream):
            return self._backward(logits, d_y, stream)

    def _backward(self, logits, d_y, stream):
        T, k, R = self.T, self.k, self.T * self.k
        at = self.row_of.long()
        # y[t] = sum over j of weight[t, j] * y_rows[row_of[t, j]]
        d_weight = (self.y_rows[at].float().view(T, k, self.d) * d_y[:, None]).sum(2)
        d_rows = (self.weight[:, :, None] * d_y[:, None]).view(R, self.d)
        g, s = _codes(R, self.d, torch.float8_e5m2)
        B.quantize_rows(d_rows, g, s, self.row_of, 1)
        d_h = torch.empty(R, self.f, device="cuda")
        B.expert_matmul(g, s, *self.w[1][2:], self.offsets, self.d, self.f, d_h)
        d_h *= self.h_q[0][:, :self.f].float() != 0  # ReLU: where the hidden activation came through
        g, s = _codes(R, self.f, torch.float8_e5m2)
        B.quantize_rows(d_h, g, s)
        d_rows = torch.empty(R, self.d, dtype=torch.bfloat16, device="cuda")
        B.expert_matmul(g, s, *self.w[0][2:], self.offsets, self.f, self.d, d_rows)
        d_x = torch.empty(T, self.d, dtype=torch.bfloat16, device="cuda")
        self.ctx.combine(d_rows, self.row_of, torch.ones_like(self.weight), T, d_x, stream=stream)
        d_logits = torch.empty_like(logits)
        self.router.route_backward(logits, self.idx, d_weight, None, d_logits)
        return d_x, d_logits


def reference(x, logits, w1, w2, top_k):
    """The same block unquantised, in float32, softmax with renormalised weights."""
    top, idx = torch.topk(logits, top_k, dim=1)
    weight = torch.softmax(top, 1)
    y = torch.zeros(x.shape, device=x.device)
    for e in range(w1.shape[0]):
        t, j = (idx == e).nonzero(as_tuple=True)
        if len(t):
            y = y.index_add(0, t, weight[t, j][:, None] * (torch.relu(x[t].float() @ w1[e].float()) @ w2[e].float()))
    return y


def run(tokens, d_model, d_ff, experts, top_k, replays=20):
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    w1, w2 = (0.02 * normal(experts, d_model, d_ff)).bfloat16(), (0.02 * normal(experts, d_ff, d_model)).bfloat16()
    x, gate = normal(tokens, d_model).bfloat16(), 0.05 * normal(d_model, experts)
    block = Block(w1, w2, gate, top_k, tokens, renormalize=True)
    logits = block.logits(x)
    y = block.forward(x, logits).float()
    want_x, want_z = x.float().requires_grad_(), logits.detach().clone().requires_grad_()
    want = reference(want_x, want_z, w1, w2, top_k)
    d_y = normal(tokens, d_model)
    d_x, d_logits = block.backward(logits, d_y)
    want_dx, want_dz = torch.autograd.grad(want, (want_x, want_z), d_y)
    off = lambda a, b: float((a.detach().float() - b.detach()).norm() / b.detach().norm())  # noqa: E731
    errors = {"y": off(y, want), "d_x": off(d_x, want_dx), "d_logits": off(d_logits, want_dz)}

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        block.forward(x, logits, stream)
    graph.replay()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(replays):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    same = torch.equal(block.y.float(), y)
    del graph
    block.close()
    return errors, 1e3 * begin.elapsed_time(end) / replays, same


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("tokens", 4096), ("d-model", 1024), ("d-ff", 4096), ("experts", 64), ("top-k", 2)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    errors, us, same = run(a.tokens, a.d_model, a.d_ff, a.experts, a.top_k)
    print("relative to float32 experts: " + ", ".join(f"{k} {v:.3g}" for k, v in errors.items()))
    print(f"forward, captured and replayed: {us:.1f} us, {a.tokens / us:.3f} M tokens/s; replays give the eager result: {same}")


if __name__ == "__main__":
    main()
