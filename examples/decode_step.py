"""One decode step, measured on the card and simulated.

The split-KV decode workload (gen.workloads.splitkv_decode) draws a batch's key
lengths and builds the tile graph of its attention.  This program runs the same
attention with the package's operators -- new keys rotated and appended to a
paged cache, queries rotated, attention over the cache -- as a captured graph on
the GPU, and simulates the tile graph on a machine record, so that the two
times stand side by side.  With --prefix P every sequence's first P keys are one
shared prefix, stored once and read once; the tile graph, which knows no
sharing, stays the same.

    python examples/decode_step.py [--batch 64] [--kv-max 32768] [--prefix 0] [--steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2607_11262_amd import api, ops
from paper_2607_11262_amd.gen import hw as H
from paper_2607_11262_amd.gen import workloads as W

MHZ = 2400


def mi355x() -> np.ndarray:
    """A record from the card's public figures (256 CUs at 2.4 GHz, 2.5
    PFLOP/s of 16-bit matrix products, 157 TFLOP/s of 32-bit vectors, 160 KiB of
    LDS a CU at 128 B a cycle, 8 TB/s); latencies of the package's H100."""
    h = H.preset("H100")
    return H.preset("H100", n_sm=256, smem_kib=160, rate_tensor=4096 * H.Q16, rate_alu=128 * H.Q16, rate_sfu=32 * H.Q16,
                    rate_gmem=64 * H.Q16, rate_l2=16384 * H.Q16, rate_dram=H.dram_q16(8_000_000, MHZ),
                    lat_l2=H.get(h, "lat_l2"), lat_dram=H.get(h, "lat_dram"))


class Decode:
    """The state of a decoding batch: the cache, its page table, and a step."""

    def __init__(self, lens, prefix, *, q_heads=32, kv_heads=8, dim=128, page=64, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        B = len(lens)
        own = [max(n - prefix, 1) for n in lens]
        per = [-(-(n + 64) // page) for n in own]  # room for 64 steps
        n_prefix, total = -(-prefix // page), -(-prefix // page) + sum(per)
        order = torch.randperm(total, generator=g, device="cuda").int()
        self.k_cache, self.v_cache = rnd(total, page, kv_heads, dim), rnd(total, page, kv_heads, dim)
        self.prefix, self.prefix_pages = prefix, order[:n_prefix].contiguous() if prefix else None
        self.pages = torch.zeros(B, max(per), dtype=torch.int32, device="cuda")
        at = n_prefix
        for b, n in enumerate(per):
            self.pages[b, :n] = order[at:at + n]
            at += n
        self.lens = torch.tensor(own, dtype=torch.int32, device="cuda")
        self.table = ops.rotary_table(max(lens) + 65, dim)
        self.q, self.k, self.v = rnd(B, q_heads, dim), rnd(B, kv_heads, dim), rnd(B, kv_heads, dim)

    def step(self):
        """One new token of every sequence: lens counts it already."""
        q = ops.append_kv(self.k, self.v, self.k_cache, self.v_cache, self.pages, self.lens, table=self.table,
                          prefix_len=self.prefix, q=self.q)
        return ops.shared_prefix_attention(q, self.k_cache, self.v_cache, self.pages, self.lens,
                                           prefix_pages=self.prefix_pages, prefix_len=self.prefix)


def measure(decode, steps):
    """Microseconds a step of a captured graph, its sequences a key longer each
    time, and the last output."""
    decode.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = decode.step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(2):  # the first of each costs its setup
        decode.lens += 1
        graph.replay()
    begin.record()
    for _ in range(steps):
        decode.lens += 1
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    return begin.elapsed_time(end) / steps * 1e3, out


def simulate(graph, record):
    """Microseconds of the graph's makespan under one record."""
    res = api.simulate(api.upload(graph), record.reshape(1, -1), 0)
    torch.cuda.synchronize()
    _, makespan, status, _ = api.to_numpy(res)
    if status[0] != api.SIM_OK:
        raise RuntimeError(f"simulation ended with status {status[0]}")
    return float(makespan[0]) / MHZ


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batch", type=int, default=64)
    p.add_argument("--kv-max", type=int, default=32768)
    p.add_argument("--prefix", type=int, default=0)
    p.add_argument("--steps", type=int, default=20)
    a = p.parse_args(argv)
    if not 1 <= a.steps <= 60:
        p.error("--steps is 1 to 60")
    graph = W.splitkv_decode(a.batch, kv_max=a.kv_max)
    lens = graph.meta["kv_lens"]
    if a.prefix >= min(lens):
        p.error(f"--prefix is below the shortest sequence, {min(lens)} keys")
    measured, out = measure(Decode(lens, a.prefix), a.steps)
    simulated = simulate(graph, mi355x())
    keys = a.prefix + sum(n - a.prefix for n in lens)
    print(f"{a.batch} sequences, {sum(lens)} keys, {keys} of them stored: measured {measured:.1f} us a step "
          f"({keys * 2 * 8 * 128 * 2 / measured / 1e3:.0f} GB/s of keys and values), "
          f"attention simulated {simulated:.1f} us")
    return dict(measured=measured, simulated=simulated, out=out)


if __name__ == "__main__":
    main()
