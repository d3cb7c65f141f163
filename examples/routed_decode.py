"""Decoding steps of a small routed network: projection with 4-bit weights, router, mixture-of-experts layer.

Each step takes the rows of a batch of tokens through `layers` blocks
    y = X P^T                          tf_q4_matvec, P in 4 bits
    A = best experts of y R^T          tf_moe_route, R the router's weights
    X = X + layer of y over A          tf_moe_layer_q4 (or tf_moe_layer with --dense)
and all launches of a step are captured into one graph.  The result is compared with the same network in 64 bits.

    python examples/routed_decode.py [--tokens 4] [--width 1024] [--hidden 768] [--experts 16] [--k 4] [--dense]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_00243_amd as tf  # noqa: E402


def quantized(weights, group):
    """A Q4Matrix of the weights (matrices x outputs x inputs) and the values that it stands for."""
    mats, rows, cols = weights.shape
    sizes = tf.tf_q4_sizes(rows, cols, tf.TF_Q4_E2M1, group, mats)
    q = tf.Q4Matrix(rows, cols, tf.TF_Q4_E2M1, group, *(torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes),
                    n_mats=mats)
    stream = torch.cuda.current_stream().cuda_stream
    tf.tf_q4_quantize(q, weights, stream)
    values = torch.empty_like(weights, dtype=torch.float32)
    tf.tf_q4_unpack(q, values, stream)
    return q, values


class Block:
    def __init__(self, args, gen):
        def normal(*shape):
            return torch.randn(*shape, device="cuda", generator=gen).div_(math.sqrt(shape[-1])).bfloat16()

        e, h, i, t = args.experts, args.width, args.hidden, args.tokens
        self.project, self.p = quantized(normal(1, h, h), 64)
        self.router = normal(e, h)
        w1, w2 = normal(e, 2 * i, h), normal(e, h, i)
        if args.dense:
            self.w1, self.w2, self.v1, self.v2 = w1, w2, w1.float(), w2.float()
        else:
            (self.w1, self.v1), (self.w2, self.v2) = quantized(w1, 32), quantized(w2, 32)
        self.plan = tf.MoePlan(e, h, i, torch.bfloat16, max_tokens=t, max_entries=t * args.k)
        self.y = torch.empty(t, h, dtype=torch.bfloat16, device="cuda")
        self.d = torch.empty_like(self.y)
        self.a = tf.DeviceCsr(t, e, torch.empty(t + 1, dtype=torch.int32, device="cuda"),
                              torch.empty(t * args.k, dtype=torch.int32, device="cuda"),
                              torch.empty(t * args.k, device="cuda"))

    def run(self, x):
        stream = torch.cuda.current_stream().cuda_stream
        tf.tf_q4_matvec(self.project, x, self.y, stream)
        scores = self.y @ self.router.t()
        tf.tf_moe_route(scores, self.a, tf.TF_ROUTE_SOFTMAX_TOP, stream=stream)
        self.plan.run(self.a, self.y, self.w1, self.w2, self.d, stream)
        return x + self.d

    def reference(self, x):
        """The block in 64 bits with the experts that `run` took for these rows."""
        y = x @ self.p[0].double().t()
        cols = self.a.colidx.view(x.shape[0], -1).long()
        scores = y @ self.router.double().t()
        share = torch.softmax(torch.gather(scores, 1, cols), 1)
        d = torch.zeros_like(x)
        for t in range(x.shape[0]):
            for q, e in enumerate(cols[t].tolist()):
                g, u = (self.v1[e].double() @ y[t]).chunk(2)
                d[t] += share[t, q] * (self.v2[e].double() @ (torch.nn.functional.silu(g) * u))
        return x + d


def main(argv=None):
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 4), ("width", 1024), ("hidden", 768), ("experts", 16), ("k", 4), ("layers", 2), ("steps", 3)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dense", action="store_true")
    args = ap.parse_args(argv)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    blocks = [Block(args, gen) for _ in range(args.layers)]
    x = torch.empty(args.tokens, args.width, dtype=torch.bfloat16, device="cuda")
    rows = []          # what goes into each block

    def step():
        del rows[:]
        z = x
        for b in blocks:
            rows.append(z)
            z = b.run(z)
        return z

    x.normal_(generator=gen)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    worst = 0.0
    for _ in range(args.steps):
        x.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        # block by block, so that a token near the border between two experts takes the same ones
        for b, z, got in zip(blocks, rows, rows[1:] + [out]):
            ref = b.reference(z.double())
            worst = max(worst, ((got.double() - ref).norm() / ref.norm()).item())
    for b in blocks:
        b.plan.close()
    print(f"{args.steps} steps of {args.layers} blocks, {args.tokens} tokens: relative error of a block {worst:.1e}")
    return worst


if __name__ == "__main__":
    sys.exit(0 if main() < 1e-2 else 1)
