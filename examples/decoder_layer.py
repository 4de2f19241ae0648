"""One decoder layer at prefill, measured on the card and simulated.

The decoder-layer workload (gen.workloads.decoder_layer) builds the tile graph of a
Llama-like layer: norm, QKV product, rotary positions, causal attention, output
product, norm, gated feed-forward.  This program runs the same layer with the
package's operators as a captured graph on the GPU, and simulates the tile graph on
a machine record, so that the two times stand side by side.  With --backward it also
measures the gradients of all weights and of the input.

    python examples/decoder_layer.py [--tokens 2048] [--hidden 4096] [--heads 32] [--kv-heads 8] [--ffn 14336] [--backward]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from decode_step import mi355x, simulate
from paper_2607_11262_amd import ops
from paper_2607_11262_amd.gen import workloads as W

DIM = 128


class Layer:
    """Weights of a layer, and a pass over a prompt."""

    def __init__(self, tokens, hidden, heads, kv_heads, ffn, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda n, k: (torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).to(torch.bfloat16)  # noqa: E731
        self.heads, self.kv_heads = heads, kv_heads
        ones = torch.ones(hidden, device="cuda", dtype=torch.bfloat16)
        self.weights = dict(norm1=ones, qkv=rnd((heads + 2 * kv_heads) * DIM, hidden), o=rnd(hidden, heads * DIM),
                            norm2=ones.clone(), gate=rnd(ffn, hidden), up=rnd(ffn, hidden), down=rnd(hidden, ffn))
        self.positions = torch.arange(tokens, device="cuda")
        self.table = ops.rotary_table(tokens, DIM)
        self.x = torch.randn((tokens, hidden), generator=g, device="cuda").to(torch.bfloat16)

    def forward(self, x, w):
        h = ops.layer_norm(x, w["norm1"], center=False)
        q, k, v = ops.linear(h, w["qkv"]).view(x.shape[0], -1, DIM).split((self.heads, self.kv_heads, self.kv_heads), 1)
        q, k = ops.rotary(q, self.positions, self.table), ops.rotary(k, self.positions, self.table)
        x = ops.linear(ops.prompt_attention(q, k, v).flatten(1), w["o"], residual=x)
        h = ops.layer_norm(x, w["norm2"], center=False)
        h = ops.linear(h, w["gate"], activation="silu", gate=ops.linear(h, w["up"]))
        return ops.linear(h, w["down"], residual=x)

    def step(self):
        with torch.no_grad():
            return self.forward(self.x, self.weights)

    def train(self):
        """The result and the gradients of its sum's input and weights."""
        x = self.x.detach().requires_grad_()
        w = {k: t.detach().requires_grad_() for k, t in self.weights.items()}
        y = self.forward(x, w)
        return y.detach(), torch.autograd.grad(y, [x, *w.values()], torch.ones_like(y))


def measure(f, steps):
    """Microseconds a pass of a captured graph, and its last result."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        f()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = f()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(2):
        graph.replay()
    begin.record()
    for _ in range(steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / steps * 1e3, out


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--hidden", type=int, default=4096)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    p.add_argument("--ffn", type=int, default=14336)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--backward", action="store_true")
    a = p.parse_args(argv)
    if a.heads * DIM != a.hidden or a.heads % a.kv_heads or a.tokens % 128:
        p.error(f"--hidden is --heads of {DIM}, --heads a multiple of --kv-heads, --tokens one of 128")
    layer = Layer(a.tokens, a.hidden, a.heads, a.kv_heads, a.ffn)
    measured, out = measure(layer.step, a.steps)
    result = dict(measured=measured, out=out)
    flops = 2 * a.tokens * a.hidden * (2 * a.hidden + 2 * a.kv_heads * DIM + 3 * a.ffn) + 2 * DIM * a.heads * a.tokens ** 2
    print(f"{a.tokens} tokens: measured {measured:.1f} us a layer ({flops / measured / 1e6:.0f} TFLOP/s)", flush=True)
    if a.backward:
        result["train"], (_, result["grads"]) = measure(layer.train, a.steps)
        print(f"with all gradients {result['train']:.1f} us", flush=True)
    graph = W.decoder_layer(a.tokens, a.hidden, a.heads, a.kv_heads, a.ffn, DIM)
    result["simulated"] = simulate(graph, mi355x())
    print(f"simulated {result['simulated']:.1f} us")
    return result


if __name__ == "__main__":
    main()
