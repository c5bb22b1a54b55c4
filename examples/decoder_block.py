"""A decoder block on one rank with both halves of the library: attention over a 4-bit paged cache, then the experts.

    python examples/decoder_block.py [--heads 64] [--kv-heads 4] [--d 4096] [--f 1536] [--experts 16] [--prompt 1000]

Random weights, plain matrix products for the projections.  Sequences are filled with prompts and then decoded token by token (a
CUDA graph of one step, whose positions and lengths move on the device); prints the device time of either."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_13057_b200 import binding as B                    # noqa: E402
from paper_2608_13057_b200.layer import Attention, MoELayer       # noqa: E402

PAGE, D = 64, 128


class Block:
    """norm, projection, attention, projection, norm, experts, norm: one residual stream in, one out."""

    def __init__(self, a, n_pages, max_tokens, g):
        dev, bf = "cuda", torch.bfloat16
        d, Hq, Hkv, E, f, k = a.d, a.heads, a.kv_heads, a.experts, a.f, 2
        rand = lambda *s: (torch.randn(*s, generator=g, device=dev) * s[-1] ** -0.5).to(bf)
        ones = torch.ones(d, dtype=bf, device=dev)
        ang = torch.arange(8192, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(D // 2, device=dev) / (D // 2))
        heads = torch.ones(D, dtype=bf, device=dev)
        self.attention = Attention(n_pages, PAGE, Hq, Hkv, D, max_tokens, cos_sin=torch.cat([ang.cos(), ang.sin()], 1).float(),
                                   q_w=heads, k_w=heads)
        self.w_in, self.w_qkv, self.w_o = ones, rand((Hq + 2 * Hkv) * D, d), rand(d, Hq * D)
        shape = B.make_shape(1, k, E, E, 1, d, f, 128)
        packed = torch.empty(B.tempo_packed_weight_bytes_bf16(shape), dtype=torch.uint8, device=dev)
        B.tempo_pack_weights_bf16(shape, rand(E, 2 * f, d), rand(E, d, f), packed)
        slots = torch.arange(E, dtype=torch.int32, device=dev)[:, None].contiguous()
        self.experts = MoELayer(max_tokens, k, E, f, rand(E, d), slots, packed, ones, post_w=ones, bf16=True)
        self.x = torch.empty(max_tokens, d, dtype=bf, device=dev)
        self.heads_out = torch.empty(max_tokens, Hq * D, dtype=bf, device=dev)

    def forward(self, r, positions, slots, page_table, lens, q_start=None, max_q=1):
        T = r.shape[0]
        x, o = self.x[:T], self.heads_out[:T]
        B.tempo_norm_in(r, self.w_in, x)
        self.attention.forward(x @ self.w_qkv.t(), positions, slots, page_table, lens, o, q_start=q_start, max_q=max_q)
        r = r + o @ self.w_o.t()
        return self.experts.forward(r, torch.empty_like(r))


def timed(f, n):
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    t0.record()
    for _ in range(n):
        f()
    t1.record()
    torch.cuda.synchronize()
    return t0.elapsed_time(t1) * 1e3 / n


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("heads", 64), ("kv-heads", 4), ("d", 4096), ("f", 1536), ("experts", 16), ("prompt", 1000), ("sequences", 4), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    n, per = a.sequences, -(-(a.prompt + a.steps + 8) // PAGE)
    block = Block(a, n * per, n * a.prompt, g)
    table = torch.randperm(n * per, generator=g, device="cuda").to(torch.int32).view(n, per)
    slot = lambda seq, t: table[seq, t // PAGE] * PAGE + (t % PAGE).to(torch.int32)

    seq = torch.arange(n, device="cuda").repeat_interleave(a.prompt)
    t = torch.arange(a.prompt, device="cuda").repeat(n)
    starts = torch.arange(n + 1, device="cuda", dtype=torch.int32) * a.prompt
    lens = torch.full((n,), a.prompt, dtype=torch.int32, device="cuda")
    r = torch.randn(n * a.prompt, a.d, generator=g, device="cuda").to(torch.bfloat16)
    prompt = lambda: block.forward(r, t.to(torch.int32), slot(seq, t), table, lens, q_start=starts, max_q=a.prompt)
    last = prompt()[a.prompt - 1::a.prompt].clone()
    print(f"{n} prompts of {a.prompt} tokens: {timed(prompt, 5):8.1f} us")

    # one decode step: the stream it reads and writes, and where each sequence stands, stay on the device
    every = torch.arange(n, device="cuda")
    stream = last

    def step():
        at = lens.clone()
        lens.add_(1)
        stream.copy_(block.forward(stream, at, slot(every, at.long()), table, lens))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())            # the prompts ran there
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    lens.fill_(a.prompt)
    stream.copy_(prompt()[a.prompt - 1::a.prompt])
    us = timed(graph.replay, a.steps)
    status = int(block.attention.status) | int(block.experts.status)
    print(f"{a.steps} steps of {n} sequences: {us:8.1f} us a step, {int(lens[0])} tokens each, status {status}")
    assert status == 0 and bool(stream.isfinite().all()) and int(lens[0]) == a.prompt + a.steps


if __name__ == "__main__":
    main()
