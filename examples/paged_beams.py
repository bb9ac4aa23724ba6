"""A beam search on the paged cache.  A prompt is appended and attended a chunk of tokens at a time; its sequence is forked into beams, which share its full pages;
at every step a token of each beam is appended and attended, with capped logits and a window behind the first rows, the logits give the next beams
(beam_select), and the pages follow them (PagedCache.fork).  Half way the cache is thinned out on its pages (PagedCache.compact).

There is no model: a token's queries, keys and values come from a table, and logits are products of the attention's output with another one.  At the end the best beam's tokens
are appended to a cache of their own, thinned out at the same step, and its rows compared with the beam's bit for bit; its last attention is compared with attention in 64 bits.
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
    ap.add_argument("--chunk", type=int, default=2048)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--vocab", type=int, default=16384)
    args = ap.parse_args()

    import torch
    import paper_2605_26678_amd as nkv

    B, T, V, H, G, d = args.beams, args.tokens, args.vocab, 8, 4, 128
    Hq, scale, dev, bf16, rows_page = H * G, d ** -0.5, "cuda:0", torch.bfloat16, nkv.PAGE_ROWS
    cap, window, prefix = 30.0, args.prompt // 2, 4
    fmt = nkv.PAGES_FP4 if args.format == "fp4" else nkv.PAGES_16BIT
    g = torch.Generator(device=dev).manual_seed(5)
    table = torch.randn(V, Hq + 2 * H, d, device=dev, generator=g).to(bf16)
    head = (torch.randn(Hq * d, V, device=dev, generator=g) * 0.2).to(bf16)
    prompt = torch.randint(V, (args.prompt,), device=dev, generator=g)
    rope = nkv.rope_table(args.prompt + T, d, device=dev)
    most = args.prompt + T
    per_unit = (most + rows_page - 1) // rows_page

    def rules(n_seqs):
        return nkv.LogitRules(cap, window, prefix=torch.full((n_seqs,), prefix, dtype=torch.int32, device=dev))

    def new_cache(n_seqs):
        # the prompt's pages once, those that the beams write, and as many again while rows are thinned out
        return nkv.PagedCache(n_seqs, H, d, nkv.DTYPE_BF16, fmt, 2 * H * (per_unit + n_seqs * (T // rows_page + 2) + n_seqs * per_unit), most)

    def attend(pages, tokens, first):
        """Tokens [sequences, n] at positions first, ..: appended and attended."""
        S, n = tokens.shape
        x, q, out = table[tokens], torch.empty(S, n, Hq, d, dtype=bf16, device=dev), torch.empty(S, n, Hq, d, dtype=bf16, device=dev)
        positions = torch.arange(first, first + n, dtype=torch.int32, device=dev).expand(S, n).contiguous()
        pages.lens.add_(n)
        nkv.pages_append(x[:, :, Hq:Hq + H], x[:, :, Hq + H:], pages, positions=positions, rope=rope, q=x[:, :, :Hq], q_out=q)
        ws = torch.empty(max(1, nkv.pages_prompt_workspace_bytes(pages, Hq, n)), dtype=torch.uint8, device=dev)
        nkv.pages_prompt_attention(q, pages, Hq, n, scale, out, None, ws, rules=rules(S))
        return q, out

    def read_prompt(cache):
        cache.reserve([args.prompt] * H + [0] * (len(cache.lens) - H))
        first = nkv.Pages(1, H, d, nkv.DTYPE_BF16, fmt, cache.pool, cache.table[:H], cache.lens[:H])
        for at in range(0, args.prompt, args.chunk):
            q, out = attend(first, prompt[None, at:at + args.chunk], at)
        return out[:, -1]

    def thin_out(cache, rows):
        """Every second row of the prompt's first half goes, of all sequences."""
        keep = torch.cat([torch.arange(0, args.prompt // 2, 2), torch.arange(args.prompt // 2, rows)]).int()
        units, n = len(cache.lens), len(keep)
        cache.compact(keep.repeat(units).to(dev), torch.arange(units + 1, device=dev) * n, [n] * units)
        return n

    # ---- the search ----
    cache = new_cache(B)
    n_pages = cache.free_pages
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    out = read_prompt(cache).expand(B, Hq, d)
    stop.record()
    torch.cuda.synchronize()
    took = start.elapsed_time(stop)
    cache.fork([0] * B, [args.prompt] * H + [0] * (B - 1) * H)
    rows, thinned = args.prompt, T // 2
    scores = torch.full((1, B), -float("inf"), device=dev)
    scores[0, 0] = 0.0                                                        # (all beams are the same one yet)
    chosen, tokens = (torch.empty(1, B, dtype=torch.int32, device=dev) for _ in range(2))
    ws = torch.empty(nkv.beam_workspace_bytes(1, B, V, B), dtype=torch.uint8, device=dev)
    said = torch.empty(B, 0, dtype=torch.int64, device=dev)
    for t in range(T):
        logits = (out.reshape(B, Hq * d) @ head)[None]
        nkv.beam_select(logits, scores, scores, chosen, tokens, ws)
        cache.fork(chosen[0].tolist(), [rows] * (B * H))
        said = torch.cat([said[chosen[0].long()], tokens[0, :, None].long()], 1)
        if t == thinned:
            rows = thin_out(cache, rows)
        rows += 1
        cache.reserve([rows] * (B * H))
        q, out = attend(cache.pages, said[:, -1:], args.prompt + t)
        out = out[:, 0]

    # ---- the best beam by itself ----
    alone = new_cache(1)
    read_prompt(alone)
    n = args.prompt
    for t in range(T):
        if t == thinned:
            n = thin_out(alone, n)
        n += 1
        alone.reserve([n] * H)
        attend(alone.pages, said[:1, t:t + 1], args.prompt + t)
    off = torch.arange(H + 1, device=dev) * rows
    first = nkv.Pages(1, H, d, nkv.DTYPE_BF16, fmt, cache.pool, cache.table[:H], cache.lens[:H])
    k, v, k1, v1 = (torch.empty(H * rows, d, dtype=bf16, device=dev) for _ in range(4))
    nkv.pages_read(k, v, off, H * rows, first)
    nkv.pages_read(k1, v1, off, H * rows, alone.pages)
    same = bool(torch.equal(k, k1) and torch.equal(v, v1))
    i = torch.arange(rows, device=dev)
    seen = (i > rows - 1 - window) | (i < prefix)
    worst = 0.0
    for h in range(H):
        z = scale * q[0, 0, h * G:(h + 1) * G].double() @ k.view(H, rows, d)[h].double().T
        z = (cap * torch.tanh(z / cap)).masked_fill(~seen, -float("inf"))
        want = torch.softmax(z, -1) @ v.view(H, rows, d)[h].double()
        worst = max(worst, float((out[0, h * G:(h + 1) * G] - want).abs().max()))
    held = n_pages - cache.free_pages
    print(f"prompt of {args.prompt} tokens in {took:.1f} ms; {B} beams of {rows} rows on {held} {args.format} pages ({B * H * ((rows + rows_page - 1) // rows_page)} if none were shared); "
          f"best score {float(scores[0, 0]):.2f}; its rows are {'those of a cache of its own' if same else 'OTHERS'}; last step off by {worst:.1e}")
    assert same and worst <= 2 * 2.0 ** -8 * max(1.0, float(v.abs().max()))
    return 0


if __name__ == "__main__":
    sys.exit(main())
