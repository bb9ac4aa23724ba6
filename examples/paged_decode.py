#!/usr/bin/env python3
"""Compress a prompt's cache, keep what is left on 4-bit (or 16-bit) pages, and decode over it.

    python examples/paged_decode.py [--format fp4|16bit] [--prompt 8192] [--ratio 0.75] [--tokens 64] [--layers 4]

For every prompt and layer: Compressor (score, budgets, selection) -> pages_load.  Then, token by token, each layer appends the
new token's key and value, rotated by its position in the text, and attends over its pages; a step of all layers is one
HIP graph, and the cache is given more pages between steps as it grows.  There is no model: queries, keys and values are synthetic.  At the end the last step is compared with attention in
64 bits over the pages' rows (pages_read), and the cache's size and a step's time are printed.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def main() -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--format", choices=("fp4", "16bit"), default="fp4")
    ap.add_argument("--prompt", type=int, default=8192)
    ap.add_argument("--prompts", type=int, default=2)
    ap.add_argument("--ratio", type=float, default=0.75)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--layers", type=int, default=4)
    args = ap.parse_args()

    import torch
    import nkv_inputs
    import paper_2605_26678_amd as nkv

    P, L, H, G, d = args.prompts, args.layers, 8, 4, 128
    Hq, scale, dev, bf16 = H * G, d ** -0.5, "cuda:0", torch.bfloat16
    fmt = nkv.PAGES_FP4 if args.format == "fp4" else nkv.PAGES_16BIT
    w = nkv_inputs.small_workload("paged_decode", L, H, d, [args.prompt] * P)
    K, V = nkv_inputs.make_kv(w, dev)
    shape = nkv.Shape(L, H, d, d, nkv.DTYPE_BF16, w.cu_seqlens)

    # the prompts' retained rows, into pages: the units of the packed rows, (prompt, layer, head), are those of P * L sequences
    comp = nkv.Compressor(shape, [args.ratio] * P)
    r = comp.run(K, V)
    kept = (r.head_off[1:] - r.head_off[:-1]).cpu()
    room = [int(n) + args.tokens + 1 for n in kept]
    cache = nkv.PagedCache(P * L, H, d, nkv.DTYPE_BF16, fmt, sum((n + nkv.PAGE_ROWS - 1) // nkv.PAGE_ROWS for n in room), max(room))
    cache.reserve(kept.tolist())
    cache.lens.copy_(kept.int())
    nkv.pages_load(r.packed_k, r.packed_v, r.head_off, comp.rows, cache.pages)

    layers, lens = cache.layers(L), cache.layer_lens                          # one Pages a layer, and what the steps count in

    g = torch.Generator(device=dev).manual_seed(7)
    qkv = torch.randn(L, P, 1, Hq + 2 * H, d, device=dev, generator=g).to(bf16)
    rope = nkv.rope_table(args.prompt + args.tokens + 1, d, device=dev)
    positions = torch.full((P, 1), args.prompt - 1, dtype=torch.int32, device=dev)
    q = torch.empty(L, P, 1, Hq, d, dtype=bf16, device=dev)
    out, lse = torch.empty(L, P, 1, Hq, d, device=dev), torch.empty(L, P, 1, Hq, device=dev)
    ws = torch.empty(nkv.pages_workspace_bytes(layers[0], Hq), dtype=torch.uint8, device=dev)

    def step():
        lens.add_(1)
        positions.add_(1)
        for l in range(L):
            x = qkv[l]
            nkv.pages_append(x[:, :, Hq:Hq + H], x[:, :, Hq + H:], layers[l], positions=positions, rope=rope, q=x[:, :, :Hq], q_out=q[l])
            nkv.pages_attention(q[l], layers[l], Hq, 1, scale, out[l], lse[l], ws)

    done = 0

    def grow():                                                               # every 32 tokens, pages for 32 more
        nonlocal done
        if done % 32 == 0:
            cache.reserve([min(int(n) + done + 32, most) for n, most in zip(kept, room)])
        done += 1

    grow()
    step()                                                                    # once outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(args.tokens // 2):
        grow()
        graph.replay()
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    timed = args.tokens - 1 - args.tokens // 2
    for _ in range(timed):
        grow()
        qkv.mul_(-1)                                                          # another token
        graph.replay()
    stop.record()
    torch.cuda.synchronize()

    # the last layer's last step against the definition, over the rows that its pages hold
    n = lens[L - 1].reshape(-1).cpu()
    off = torch.zeros(P * H + 1, dtype=torch.int64)
    off[1:] = torch.cumsum(n, 0)
    rows = int(off[-1])
    k, v = (torch.empty(rows, d, dtype=bf16, device=dev) for _ in range(2))
    nkv.pages_read(k, v, off.to(dev), rows, layers[L - 1])
    worst = 0.0
    for u in range(P * H):
        p, h = divmod(u, H)
        a, b = int(off[u]), int(off[u + 1])
        z = scale * q[L - 1, p, 0, h * G:(h + 1) * G].double() @ k[a:b].double().T
        want = torch.softmax(z, -1) @ v[a:b].double()
        worst = max(worst, float((out[L - 1, p, 0, h * G:(h + 1) * G] - want).abs().max()))
    held, full = cache.pool.numel(), 2 * 2 * d * L * H * P * args.prompt
    print(f"{P} prompts of {args.prompt} tokens, {L} layers: {args.format} pages hold {held / 2**20:.1f} MiB of a {full / 2**20:.1f} MiB cache; "
          f"{timed} steps, {start.elapsed_time(stop) / timed * 1e3:.1f} us each ({L} layers' append and attention); last step off by {worst:.1e}")
    assert worst <= 1e-5 * max(1.0, float(v.abs().max()))
    return 0


if __name__ == "__main__":
    sys.exit(main())
