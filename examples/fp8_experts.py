"""A mixture-of-experts block with its experts held in 8-bit floating point, as a program serves it, fine-tunes its router and trains its experts.

    python examples/fp8_experts.py [--tokens 4096] [--d-model 1024] [--d-ff 4096] [--experts 64] [--top-k 2] [--train]

Forward, six calls of the library: route, group the rows by expert, quantise the hidden states on their way to the experts, the two
products (the hidden activation goes from one to the other in 8 bits), combine.  Backward, with the quantisation taken as the identity:
the gradient of the hidden states through the transposed weights, rows in e5m2, that of the router's logits and, for whoever asks, those of the experts'
matrices from the rows and hidden activations that the forward kept in 8 bits (the optimizer's master weights are the caller's, as is quantising them again).
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
    """w1 [E, d, f], w2 [E, f, d]: quantised here, once, in both orientations.  gate [d, E] float32.  train: what the forward keeps gets scales that
    are powers of two, with which the gradients of the matrices take a third of the products."""

    def __init__(self, w1, w2, gate, top_k, max_tokens, train=False, **router):
        self.E, self.d, self.f = w1.shape
        self.k, self.T, self.gate, self.train = top_k, max_tokens, gate, train
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
        B.quantize_rows(x, *self.x_q, self.row_of, self.k, stream, pow2=self.train)
        B.expert_matmul(*self.x_q, w1, s1, self.offsets, self.d, self.f, *self.h_q, relu=True, stream=stream, pow2=self.train)
        B.expert_matmul(*self.h_q, w2, s2, self.offsets, self.f, self.d, self.y_rows, stream=stream)
        self.ctx.combine(self.y_rows, self.row_of, self.weight, self.T, self.y, stream=stream)
        return self.y

    def backward(self, logits, d_y, stream=None, d_w=None):
        """d_y [T, d] float32, its elements wherever they lie, after forward() on the same logits -> (d_x through the experts [T, d] bf16, d_logits [T, E]), on `stream` or
        torch's current one, like forward(): torch's operations and the library's one behind the other.  d_w: (d_w1 [E, d, f], d_w2 [E, f, d]), to which the
        gradients of the matrices are added."""
        stream = stream or torch.cuda.current_stream()
        with torch.cuda.stream(stream):
            return self._backward(logits, d_y, d_w)

    def _add_gradient(self, rows, d_rows, d_w):
        need = B.expert_weight_gradient_workspace_bytes(len(d_rows), *d_w.shape)
        workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        B.expert_weight_gradient(*rows, d_rows, self.offsets, d_w, add=d_w, pow2=self.train, workspace=workspace)

    def _backward(self, logits, d_y, d_w):
        R = self.T * self.k
        new = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        d_y = d_y.contiguous()  # the gradient of a sum over tokens is one row for all of them, which the library's calls do not take
        # y[t] = sum over j of weight[t, j] * y_rows[row_of[t, j]]
        d_weight, g, values = new(self.T, self.k, dtype=torch.float32), _codes(R, self.d, torch.float8_e5m2), new(R, self.d) if d_w else None
        B.combine_rows_backward(d_y, self.y_rows, self.row_of, self.weight, values, d_weight, *g)
        if d_w:
            self._add_gradient(self.h_q, values, d_w[1])
        d_h = new(R, self.f, dtype=torch.float32)
        B.expert_matmul(*g, *self.w[1][2:], self.offsets, self.d, self.f, d_h)
        g, values = _codes(R, self.f, torch.float8_e5m2), new(R, self.f) if d_w else None
        B.relu_backward(d_h, self.h_q[0], values, *g)
        if d_w:
            self._add_gradient(self.x_q, values, d_w[0])
        d_rows, d_x, d_logits = new(R, self.d), new(self.T, self.d), torch.empty_like(logits)
        B.expert_matmul(*g, *self.w[0][2:], self.offsets, self.f, self.d, d_rows)
        B.combine_rows(d_rows, self.row_of, d_x)
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


def run(tokens, d_model, d_ff, experts, top_k, replays=20, train=False):
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    w1, w2 = (0.02 * normal(experts, d_model, d_ff)).bfloat16(), (0.02 * normal(experts, d_ff, d_model)).bfloat16()
    x, gate = normal(tokens, d_model).bfloat16(), 0.05 * normal(d_model, experts)
    block = Block(w1, w2, gate, top_k, tokens, train=train, renormalize=True)
    logits = block.logits(x)
    y = block.forward(x, logits).float()
    leaves = [t.detach().float().requires_grad_() for t in (x, logits, w1, w2)]
    want = reference(*leaves, top_k)
    d_y, d_w = normal(tokens, d_model), (torch.zeros(w1.shape, device="cuda"), torch.zeros(w2.shape, device="cuda"))
    got = *block.backward(logits, d_y, d_w=d_w), *d_w
    gradients = torch.autograd.grad(want, leaves, d_y)
    off = lambda a, b: float((a.detach().float() - b.detach()).norm() / b.detach().norm())  # noqa: E731
    errors = {"y": off(y, want)} | {n: off(a, b) for n, a, b in zip(("d_x", "d_logits", "d_w1", "d_w2"), got, gradients)}

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
    p.add_argument("--train", action="store_true", help="keep rows and hidden activations with scales that are powers of two")
    a = p.parse_args()
    errors, us, same = run(a.tokens, a.d_model, a.d_ff, a.experts, a.top_k, train=a.train)
    print("relative to float32 experts: " + ", ".join(f"{k} {v:.3g}" for k, v in errors.items()))
    print(f"forward, captured and replayed: {us:.1f} us, {a.tokens / us:.3f} M tokens/s; replays give the eager result: {same}")


if __name__ == "__main__":
    main()
