"""A mixture-of-experts layer on one rank, decode and prefill batches: norm, router, experts, norm with the residual sum.

    python examples/moe_layer.py [--experts 128] [--local 16] [--d 4096] [--f 1536] [--topk 8]

Random weights; prints the device time of a layer for batches from one token to a few thousand (CUDA graph of consecutive
passes) and checks one small batch against plain torch."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_13057_b200 import binding as B                    # noqa: E402
from paper_2608_13057_b200.layer import MoELayer                  # noqa: E402


def fp8(G, n, k, g):
    """e4m3 codes [G, n, k] and power-of-two scales of 128x128 blocks, of N(0, 0.02) weights."""
    q = torch.empty(G, n, k, dtype=torch.uint8, device="cuda")
    s = torch.empty(G, n // 128, k // 128, device="cuda")
    for e in range(G):
        w = (torch.randn(n // 128, 128, k // 128, 128, generator=g, device="cuda") * 0.02)
        s[e] = torch.exp2(torch.ceil(torch.log2(w.abs().amax(dim=(1, 3)) / 448)))
        q[e] = (w / s[e][:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(n, k)
    return q, s


def plain(layer, weights, r):
    """The layer in 64 bits for a few tokens (this rank's experts only)."""
    (q13, s13), (q2, s2) = weights
    norm = lambda v, w: v / torch.sqrt((v * v).mean(1, keepdim=True) + layer.eps) * w.double()
    x = norm(r.double(), layer.norm_w).bfloat16().double()
    p = torch.softmax(x @ layer.w_router.double().t(), 1)
    w, ids = torch.topk(p, layer.k, dim=1)
    w = w / w.sum(1, keepdim=True)
    y = torch.zeros_like(x)
    deq = lambda q, s: q.view(torch.float8_e4m3fn).double() * s.double().repeat_interleave(128, 0).repeat_interleave(128, 1)
    for e in range(layer.G_max):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if t.numel():
            gate, up = (x[t] @ deq(q13[e], s13[e]).t()).chunk(2, 1)
            y.index_add_(0, t, (gate * torch.sigmoid(gate) * up) @ deq(q2[e], s2[e]).t() * w[t, j][:, None])
    return r.double() + norm(y, layer.post_w)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--experts", type=int, default=128)
    ap.add_argument("--local", type=int, default=16)
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--f", type=int, default=1536)
    ap.add_argument("--topk", type=int, default=8)
    a = ap.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)
    E, G, d, f, k = a.experts, a.local, a.d, a.f, a.topk
    weights = fp8(G, 2 * f, d, g), fp8(G, d, f, g)
    shape = B.make_shape(1, k, E, G, 1, d, f, 128)
    packed = torch.empty(B.tempo_packed_weight_bytes(shape), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.tempo_pack_weights(shape, weights[0][0], weights[0][1], weights[1][0], weights[1][1], packed, status)
    replica_map = torch.full((E, 1), -1, dtype=torch.int32, device="cuda")
    replica_map[:G, 0] = torch.arange(G, dtype=torch.int32, device="cuda")
    ones = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    w_router = (torch.randn(E, d, generator=g, device="cuda") * 0.02).bfloat16()
    layer = MoELayer(2048, k, G, f, w_router, replica_map, packed, ones, post_w=ones, next_w=ones)

    r = torch.randn(8, d, generator=g, device="cuda")
    out = layer.forward(r, torch.empty_like(r))
    ref = plain(layer, weights, r)
    err = float((out.double() - ref).norm() / ref.norm())
    print(f"8 tokens against 64 bits: relative error {err:.1e}, status {int(layer.status.item())}")
    assert err < 1e-2

    for T in (1, 8, 64, 65, 256, 2048):
        r = torch.randn(T, d, generator=g, device="cuda").bfloat16()
        x_next = torch.empty_like(r)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())       # r is drawn there
        with torch.cuda.stream(side):
            layer.forward(r, torch.empty_like(r), x_next)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        n = 20
        r_out = torch.empty_like(r)
        with torch.cuda.graph(graph, stream=side):
            for _ in range(n):
                layer.forward(r, r_out, x_next)
        graph.replay()
        torch.cuda.synchronize()
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        for _ in range(5):
            graph.replay()
        t1.record()
        torch.cuda.synchronize()
        local = int((layer.replica_map[layer.topk_ids[:T].long(), 0] >= 0).sum())
        print(f"{T:5d} tokens, {local:5d} (token, expert) pairs here: {t0.elapsed_time(t1) * 1e3 / (5 * n):8.1f} us a layer")


if __name__ == "__main__":
    main()
