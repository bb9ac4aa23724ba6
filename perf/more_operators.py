"""More operators on the paged cache and what they are measured on: attention of a prompt's chunk (or of single tokens) with
rules for its logits, copies of pages, compaction of rows, and beam search's selection.

Pages hold the rows of unit u = s * H + h (sequence s, KV head h), 64 on each: ``table[u][j]`` is the page of the unit's rows
64 j .. 64 j + 63, ``lens[u]`` how many rows there are.  A page is bytes of one of two formats, D the head dim:

* "16bit": K [64][D], V [64][D] in the type of the rows;
* "fp4": K codes [64][D / 2], V codes [16 row quads][D / C chunks][4 rows][C / 2] (C = 4, 8, 16 dims for D <= 64, 128, 256),
  K scales [D / 32 blocks][16][4]: of row 16 t + r at [b][r][t], V scales [4][D / 32][4][4]: of row 16 t + 4 g + i at
  [g][b][t][i].  A code is 4 bits, the lower dim in the lower half: a sign and the number of one of 0, 0.5, 1, 1.5, 2, 3, 4, 6;
  a block of 32 dims of a row has the factor 2^(scale - 127).

* attention: token t of the n newest of a sequence stands on row r = lens[u] - n + t of its unit and sees the rows i <= r (a
  window w > 0: i > r - w of them) and, whatever r and w, the rows i < prefix[s]; with z_i = scale <q, k_i>, capped to
  cap * tanh(z_i / cap) where there is a cap, less slope[head] * |r - i|, out = sum_i softmax(z)_i v_i in the rows' type, lse =
  log sum_i exp(z_i);
* copy: page src[i] to page dst[i];
* compact: rows kept_idx[off[u] .. off[u + 1] - 1] of unit u become rows 0, 1, .. of the unit on pages of another table;
* beam: of every prompt's candidates (beam b, token t) those with the n_out largest scores[b] + logits[b][t] - log sum exp
  logits[b], largest first, of equal ones the lower beam, then the lower token.

``own`` False: plain torch operations.  ``own`` True: the calls of the package.
"""
from __future__ import annotations

import math

import torch

own = False

ROWS = 64
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ----------------------------------------------------------------------------------------------------------------------------

def listed():
    f = dict(path="attend", dtype="bf16", fmt="16bit", H=8, G=4, d=128, cap=0.0, window=0, slopes=False, prefix=0)
    p = dict(dtype="bf16", fmt="fp4", H=8, d=128)
    return [
        # the last chunk of the benchmark's 32k-token prompt in one layer, over everything before it: all products
        dict(f, name="chunk_32k", S=1, n=2048, held=30720),
        # prompts of a ragged batch from their first token on, capped logits and a sliding window behind the first rows, 4-bit pages
        dict(f, name="prompts_cap_window_fp4", S=3, n=2731, held=0, fmt="fp4", cap=50.0, window=1024, prefix=4),
        # short prompts behind an image or an instruction that every token sees, a small model's head dim, distances, an odd length
        dict(f, name="prefix_slopes_d64", S=8, n=509, held=130, d=64, G=3, slopes=True, prefix=300, dtype="fp16"),
        # a decode step of a serving batch: one token each, capped logits, a window that leaves a part of the cache
        dict(f, name="token_cap_window_batch", S=32, n=1, held=8192, G=8, fmt="fp4", cap=30.0, window=4096, prefix=4),
        # one token of one sequence: all latency
        dict(f, name="token_slopes", S=1, n=1, held=1024, slopes=True),
        # a beam search's new beams of one prompt get pages of their own for their last, unfinished ones
        dict(p, name="copy_tails_layer", path="copy", S=8, pages=1),
        # the same in all 36 layers at once, and 16 bits: what has been generated since the prompt moves as a whole
        dict(p, name="copy_all_layers_16bit", path="copy", S=36 * 4, pages=3, fmt="16bit"),
        # a layer's cache of a ragged batch is thinned out
        dict(p, name="compact_layer_ragged", path="compact", S=8, held=2048, share=0.5),
        # the benchmark's 36 layers of a 32k-token prompt, of which a quarter was left, a second time
        dict(p, name="compact_qwen4b_32k", path="compact", S=36, held=8192, share=0.6, fmt="16bit"),
        # four beams of one prompt, fp32 logits: all latency
        dict(name="beam_one_prompt", path="beam", P=1, B=4, V=32768, n_out=8, dtype="fp32", pad=0),
        # a serving batch, a large vocabulary
        dict(name="beam_batch", path="beam", P=16, B=8, V=131072, n_out=16, dtype="bf16", pad=0),
        # an odd vocabulary in padded rows
        dict(name="beam_odd_padded", path="beam", P=5, B=5, V=50021, n_out=10, dtype="fp16", pad=27),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    path = rng.choice(["attend", "attend", "attend", "copy", "compact", "beam", "beam"])
    if path == "beam":
        B = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
        c = dict(path=path, P=_log_int(rng, 1, 64), B=B, V=_log_int(rng, 50, 200000), n_out=rng.choice([B, 2 * B, min(64, 2 * B + 1)]),
                 dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, rng.randint(1, 64)]))
        while c["P"] * B * c["V"] > 16 << 20:
            c["P"], c["V"] = max(1, c["P"] * 2 // 3), max(50, c["V"] * 9 // 10)
        return c
    c = dict(path=path, S=_log_int(rng, 1, 64), H=rng.choice([1, 2, 4, 8, 8, 32]), d=rng.choice([64, 64, 96, 128, 128, 128, 192, 256]),
             dtype=rng.choice(["bf16", "bf16", "fp16"]), fmt=rng.choice(["fp4", "16bit"]))
    if path == "copy":
        c["pages"] = _log_int(rng, 1, 16)
        while c["S"] * c["H"] * c["pages"] * c["d"] > 3 * 36 * 32 * 128:
            c["S"], c["pages"] = max(1, c["S"] * 2 // 3), max(1, c["pages"] * 3 // 4)
        return c
    if path == "compact":
        c["held"], c["share"] = _log_int(rng, 1, 16384), rng.choice([0.1, 0.5, 0.6, 0.9, 1.0])
        while c["S"] * c["H"] * c["held"] * c["d"] > 256 << 20:
            c["S"], c["held"] = max(1, c["S"] * 2 // 3), max(1, c["held"] * 3 // 4)
        return c
    c["G"] = rng.choice([1, 2, 3, 4, 4, 6, 8, 16] if c["H"] < 32 else [1, 2])
    c["n"] = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 17, 4096), _log_int(rng, 17, 4096)])
    c["held"] = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 1, 32768)])
    c["cap"] = rng.choice([0.0, 0.0, 20.0, 50.0])
    c["window"] = rng.choice([0, 0, _log_int(rng, 1, 4096)])
    c["slopes"] = rng.random() < 0.3
    c["prefix"] = rng.choice([0, 0, 4, _log_int(rng, 1, c["n"] + c["held"])])
    while c["S"] * c["H"] * c["G"] * c["n"] * (c["n"] + c["held"]) * c["d"] > 120 << 30 or c["S"] * c["H"] * (c["n"] + c["held"]) * c["d"] > 192 << 20:
        if c["S"] > 1:
            c["S"] = max(1, c["S"] * 2 // 3)
        else:
            c["n"], c["held"] = max(1, c["n"] * 3 // 4), c["held"] * 3 // 4
    return c


# ---- inputs -------------------------------------------------------------------------------------------------------------------------------

def page_bytes(d, fmt):
    return 2 * ROWS * d * 2 if fmt == "16bit" else ROWS * d + 2 * ROWS * d // 32


def _generator(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFFFFFF)
    return g


def _lens(case):
    """Rows of every unit, part of the case and not of the seed: what the heads' uneven budgets left, and the new tokens."""
    S, H = case["S"], case["H"]
    host = torch.Generator()
    host.manual_seed(20270)
    share = torch.rand(S, H, generator=host) + 0.25
    share = share / share.mean(-1, keepdim=True) * (0.6 + 0.4 * torch.rand(S, 1, generator=host))
    if case["path"] == "copy":                            # rows on the last page; those before it are full
        return case["pages"] * ROWS - ROWS + 1 + (share * 1000003).long().reshape(-1) % ROWS
    if case["path"] == "attend" and case["n"] > 1:        # a prompt being read: nothing has been evicted
        held = case["held"] - (torch.arange(S) * 37) % max(1, case["held"] // 2 + 1)
        return (held[:, None].expand(S, H) + case["n"]).reshape(-1)
    return (share.clamp(max=1.0) * case["held"]).long().clamp(min=1 - case.get("n", 0)).reshape(-1) + case.get("n", 0)


def _tables(needs):
    """Pages of their own, somewhere in one pool, for units that need so many: ([table], pages of the pool)."""
    host = torch.Generator()
    host.manual_seed(20271)
    total = int(sum(int(n.sum()) for n in needs))
    order, at, tables = torch.randperm(total + 3, generator=host).to(torch.int32), 0, []
    for need in needs:
        width = int(need.max()) + 1
        table = torch.full((need.numel(), width), -1, dtype=torch.int32)
        mine = int(need.sum())
        table[torch.arange(width)[None, :] < need[:, None]] = order[at:at + mine]
        at += mine
        tables.append(table)
    return tables, total + 3


def _pow2(e):
    """2^e as fp32, exactly."""
    return ((e + 127) << 23).view(torch.float32)


def _to_codes(x):
    """Codes (uint8, one per value) and scales of fp32 x [..., D]: the smallest power of two that leaves a block's largest magnitude
    under 7, the nearest code."""
    b = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))
    s = torch.where(m == 0, torch.full_like(e, -126), torch.where(m >= 0.875, e - 2, e - 3)).clamp(-126, 126)
    y = b.abs() * _pow2(-s)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    return (code + 8 * torch.signbit(b)).to(torch.uint8).flatten(-2), (s.squeeze(-1) + 127).to(torch.uint8)


def _chunk(d):
    return 4 if d <= 64 else 8 if d <= 128 else 16


def _to_pages(k, v, fmt):
    """Bytes [N, page] of k, v [N, 64, D] in the rows' type."""
    N, _, D = k.shape
    if fmt == "16bit":
        return torch.stack([k, v], 1).reshape(N, -1).view(torch.uint8)
    (kc, ks), (vc, vs) = _to_codes(k.float()), _to_codes(v.float())
    kc, vc = (c[..., 0::2] | c[..., 1::2] << 4 for c in (kc, vc))
    C, nb = _chunk(D), D // 32
    vc = vc.reshape(N, 16, 4, D // C, C // 2).transpose(2, 3)
    ks = ks.reshape(N, 4, 16, nb).permute(0, 3, 2, 1)
    vs = vs.reshape(N, 4, 4, 4, nb).permute(0, 2, 4, 1, 3)
    return torch.cat([t.reshape(N, -1) for t in (kc, vc, ks, vs)], dim=1)


def _pool(case, g, table, n_pages):
    """The pool: rows as keys are (a mean direction a unit, a few strong dims, noise) and values on the table's pages, ones (NaN) on the others."""
    d, dt = case["d"], DTYPES[case["dtype"]]
    pool = torch.full((n_pages, page_bytes(d, case["fmt"])), 255, dtype=torch.uint8, device="cuda")
    mean = torch.randn(table.shape[0], 1, d, device="cuda", generator=g)
    mean[..., : max(1, d // 32)] *= 4.0
    unit, slot = (table >= 0).nonzero(as_tuple=True)
    page = table[unit, slot].long().cuda()
    unit = unit.cuda()
    at_once = max(1, (32 << 20) // (ROWS * d))
    for i in range(0, page.numel(), at_once):
        u = unit[i:i + at_once]
        k = torch.randn(u.numel(), ROWS, d, device="cuda", generator=g) + 0.7 * mean[u]
        v = torch.randn(u.numel(), ROWS, d, device="cuda", generator=g) + 0.3 * mean[u]
        pool[page[i:i + at_once]] = _to_pages(k.to(dt), v.to(dt), case["fmt"])
    return pool


def _offsets(counts):
    off = torch.zeros(counts.numel() + 1, dtype=torch.int64)
    off[1:] = torch.cumsum(counts, 0)
    return off


def prepare(case, seed):
    g, path = _generator(seed, 11), case["path"]
    f = dict(device="cuda", generator=g)
    if path == "beam":
        P, B, V, K, dt = case["P"], case["B"], case["V"], case["n_out"], DTYPES[case["dtype"]]
        # logits as a model's: wide noise, a few tokens well above it, some banned
        x = 2.0 * torch.randn(P, B, V + case["pad"], **f)
        x += 6.0 * (torch.rand(P, B, V + case["pad"], **f) < 8.0 / V) * torch.rand(P, B, V + case["pad"], **f)
        x[..., V // 3:V // 3 + 2] = -math.inf
        scores = -8.0 * torch.rand(P, B, **f)
        if B > 2:
            scores[0, B - 1] = -math.inf                  # a beam that is not there
        return dict(path=path, P=P, B=B, V=V, n_out=K, logits=x.to(dt)[..., :V], scores=scores,
                    out_scores=torch.empty(P, K, dtype=torch.float32, device="cuda"),
                    out_beams=torch.empty(P, K, dtype=torch.int32, device="cuda"), out_tokens=torch.empty(P, K, dtype=torch.int32, device="cuda"))
    S, H, d, dt = case["S"], case["H"], case["d"], DTYPES[case["dtype"]]
    lens = _lens(case)
    need = (lens + ROWS - 1) // ROWS
    s = dict(path=path, S=S, H=H, d=d, dtype=dt, fmt=case["fmt"], lens=lens.to(torch.int32).cuda())
    if path == "attend":
        (table,), n_pages = _tables([need])
        n, Hq = case["n"], H * case["G"]
        s.update(n=n, Hq=Hq, scale=1.0 / math.sqrt(d), cap=case["cap"], window=case["window"], slopes=None, prefix=None,
                 q=(1.5 * torch.randn(S, n, Hq, d, **f)).to(dt), attn=torch.empty(S, n, Hq, d, dtype=dt, device="cuda"),
                 lse=torch.empty(S, n, Hq, dtype=torch.float32, device="cuda"))
        if case["slopes"]:
            s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, Hq + 1, dtype=torch.float64) / Hq)).float().cuda()
        if case["prefix"]:
            s["prefix"] = (case["prefix"] - (torch.arange(S) * 5) % max(1, case["prefix"] // 2)).to(torch.int32).cuda()
        s.update(table=table.cuda(), pool=_pool(case, g, table, n_pages))
        return s
    if path == "copy":
        # what the new sequences hold is what others hold; they have pages of their own for it
        (table, new), n_pages = _tables([need, need])
        pool = _pool(case, g, table, n_pages)
        host = torch.Generator()
        host.manual_seed(int(seed))
        order = torch.randperm(int(need.sum()), generator=host)
        last = torch.where(lens % ROWS == 0, ROWS, lens % ROWS) + (need - 1) * ROWS
        off = _offsets(last)
        rows = int(off[-1])
        s.update(table=new.cuda(), pool=pool, src=table[table >= 0][order].cuda(), dst=new[new >= 0][order].cuda())
    else:
        kept, counts = _kept(case, lens, seed)
        new_need = (counts + ROWS - 1) // ROWS
        (table, new), n_pages = _tables([need, new_need])
        off = _offsets(counts)
        rows = int(off[-1])
        s.update(table=new.cuda(), pool=_pool(case, g, table, n_pages), old_table=table.cuda(), old_lens=s["lens"], kept=kept.cuda(),
                 lens=counts.to(torch.int32).cuda())
    s.update(head_off=off.cuda(), rows=rows, k_back=torch.empty(rows, d, dtype=dt, device="cuda"), v_back=torch.empty(rows, d, dtype=dt, device="cuda"))
    return s


def _counts(case, lens):
    return (lens.double() * case["share"]).ceil().long()


def _kept(case, lens, seed):
    """Row numbers (ascending) that stay of every unit: the first four, the newest eighth, and the best of the others by a number each."""
    host = torch.Generator()
    host.manual_seed(int(seed))
    counts = _counts(case, lens)
    most = max(1, int(lens.max()))
    i = torch.arange(most)[None, :]
    score = torch.rand(lens.numel(), most, generator=host)
    score = torch.where((i < 4) | (i >= lens[:, None] * 7 // 8), 2.0, score)
    score = torch.where(i < lens[:, None], score, -1.0)
    order = torch.argsort(score, dim=1, descending=True, stable=True)
    order = torch.where(i < counts[:, None], order, most).sort(1).values
    return order[order < most].to(torch.int32), counts


# ---- plain form ---------------------------------------------------------------------------------------------------------------------------

def _values(code, scale):
    magnitude = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=code.device)[code.int()]
    return (magnitude.unflatten(-1, (-1, 32)) * _pow2(scale.int() - 127)[..., None]).flatten(-2)


def _cached(s, table):
    """All units' pages as fp32 K, V [units, width * 64, D]."""
    D, nb, C = s["d"], s["d"] // 32, _chunk(s["d"])
    b = s["pool"][table.clamp(min=0).long()]
    units, width = b.shape[:2]
    if s["fmt"] == "16bit":
        kv = b.view(s["dtype"]).reshape(units, width, 2, ROWS, D)
        return kv[:, :, 0].reshape(units, -1, D).float(), kv[:, :, 1].reshape(units, -1, D).float()
    kc, vc, ks, vs = b.split([ROWS * D // 2, ROWS * D // 2, 2 * D, 2 * D], dim=-1)
    vc = vc.reshape(units, width, 16, D // C, 4, C // 2).transpose(3, 4)
    ks = ks.reshape(units, width, nb, 16, 4).permute(0, 1, 4, 3, 2)
    vs = vs.reshape(units, width, 4, nb, 4, 4).permute(0, 1, 4, 2, 5, 3)
    k, v = (_values(torch.stack([c & 15, c >> 4], -1).flatten(-2), x.reshape(units, width * ROWS, nb))
            for c, x in ((kc.reshape(units, width * ROWS, D // 2), ks), (vc.reshape(units, width * ROWS, D // 2), vs)))
    return k, v


def _as_rows(x, s):
    """fp32 values in the rows' type."""
    top = torch.finfo(s["dtype"]).max
    return (x.clamp(-top, top) if s["fmt"] == "fp4" else x).to(s["dtype"])


def _plain_attend(s):
    S, n, Hq, D, H = s["S"], s["n"], s["Hq"], s["d"], s["H"]
    k, v = _cached(s, s["table"])
    units, rows, G = k.shape[0], k.shape[1], Hq // H
    x = s["q"].float().reshape(S, n, H, G, D).transpose(1, 2).reshape(units, n * G, D)
    row = torch.arange(rows, device=k.device)
    there = row < s["lens"][:, None]
    k, v = torch.where(there[..., None], k, 0.0), torch.where(there[..., None], v, 0.0)
    at = (s["lens"][:, None] - n + torch.arange(n, device=k.device).repeat_interleave(G))[..., None]   # the token's own row
    seen = row <= at
    if s["window"]:
        seen = seen & (row > at - s["window"])
    if s["prefix"] is not None:
        seen = seen | (row < s["prefix"].repeat_interleave(H)[:, None, None])
    seen = seen & there[:, None] & (at >= 0)
    z = s["scale"] * torch.matmul(x, k.transpose(1, 2))
    if s["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    if s["slopes"] is not None:
        z = z - s["slopes"].reshape(1, H, 1, G).expand(S, H, n, G).reshape(units, n * G, 1) * (at - row).abs()
    z = torch.where(seen, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(z - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    back = lambda t: t.reshape(S, H, n, G, -1).transpose(1, 2).reshape(S, n, Hq, -1)  # noqa: E731
    return dict(attn=back(o).to(s["dtype"]), lse=back(lse)[..., 0])


def _plain_beam(s):
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    value = s["scores"].double()[..., None] + (x - lse)
    value = torch.where(torch.isfinite(value), value, -math.inf).flatten(1)
    best, at = torch.sort(value, dim=1, descending=True, stable=True)
    best, at = best[:, :s["n_out"]], at[:, :s["n_out"]]
    missing = s["n_out"] - best.shape[1]
    if missing > 0:
        best, at = torch.nn.functional.pad(best, (0, missing), value=-math.inf), torch.nn.functional.pad(at, (0, missing))
    none = best == -math.inf
    return dict(scores=best.float(), beams=torch.where(none, -1, at // s["V"]).int(), tokens=torch.where(none, -1, at % s["V"]).int())


def _plain(s):
    if s["path"] == "beam":
        return _plain_beam(s)
    if s["path"] == "attend":
        return _plain_attend(s)
    unit = torch.repeat_interleave(s["head_off"][1:] - s["head_off"][:-1], output_size=s["rows"])
    if s["path"] == "copy":
        s["pool"][s["dst"].long()] = s["pool"][s["src"].long()]
        row = torch.arange(s["rows"], device=unit.device) - s["head_off"][unit]
        k, v = _cached(s, s["table"])
    else:
        row = s["kept"].long()
        k, v = _cached(s, s["old_table"])
    return dict(k=_as_rows(k[unit, row], s), v=_as_rows(v[unit, row], s))


# ---- the package's calls ------------------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2605_26678_amd as nkv
    codes = {torch.bfloat16: nkv.DTYPE_BF16, torch.float16: nkv.DTYPE_F16, torch.float32: nkv.DTYPE_F32}
    if s["path"] == "beam":
        if "ws" not in s:
            s["ws"] = torch.empty(nkv.beam_workspace_bytes(s["P"], s["B"], s["V"], s["n_out"]), dtype=torch.uint8, device="cuda")
        nkv.beam_select(s["logits"], s["scores"], s["out_scores"], s["out_beams"], s["out_tokens"], s["ws"])
        return dict(scores=s["out_scores"], beams=s["out_beams"], tokens=s["out_tokens"])
    if "pages" not in s:                 # the handles and the scratch that a program keeps
        of = (s["S"], s["H"], s["d"], codes[s["dtype"]], nkv.PAGES_FP4 if s["fmt"] == "fp4" else nkv.PAGES_16BIT, s["pool"])
        s["pages"] = nkv.Pages(*of, s["table"], s["lens"])
        if s["path"] == "compact":
            s["old"] = nkv.Pages(*of, s["old_table"], s["old_lens"])
        if s["path"] == "attend":
            s["rules"] = nkv.LogitRules(cap=s["cap"], window=s["window"], slopes=s["slopes"], prefix=s["prefix"])
            s["ws"] = torch.empty(nkv.pages_prompt_workspace_bytes(s["pages"], s["Hq"], s["n"]), dtype=torch.uint8, device="cuda")
    pages = s["pages"]
    if s["path"] == "attend":
        nkv.pages_prompt_attention(s["q"], pages, s["Hq"], s["n"], s["scale"], s["attn"], s["lse"], s["ws"], rules=s["rules"])
        return dict(attn=s["attn"], lse=s["lse"])
    if s["path"] == "copy":
        nkv.pages_copy(s["src"], s["dst"], pages)
    else:
        nkv.pages_compact(s["kept"], s["head_off"], s["rows"], s["old"], pages)
    nkv.pages_read(s["k_back"], s["v_back"], s["head_off"], s["rows"], pages)
    return dict(k=s["k_back"], v=s["v_back"])


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------------------

def work(case):
    """Inputs read once and outputs written once; the products of attention for the rows that a token sees."""
    if case["path"] == "beam":
        size = 4 if case["dtype"] == "fp32" else 2
        n = case["P"] * case["B"] * case["V"]
        return {"bytes": n * size + case["P"] * (4 * case["B"] + 12 * case["n_out"]), "flops": 4 * n}
    S, H, d = case["S"], case["H"], case["d"]
    held = 4 * d if case["fmt"] == "16bit" else d + d // 16                # a row's K and V in the cache
    lens = _lens(case)
    if case["path"] == "copy":
        rows = int(lens.sum())
        pages = int(((lens + ROWS - 1) // ROWS).sum())
        return {"bytes": pages * (2 * ROWS * held + 8) + rows * 4 * d, "flops": 0}
    if case["path"] == "compact":
        rows = int(_counts(case, lens).sum())
        return {"bytes": rows * (2 * held + 4 + 4 * d), "flops": 0}
    n, G = case["n"], case["G"]
    at = lens[:, None] - n + torch.arange(n)
    first = (at - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(at)
    front = torch.zeros(S, dtype=torch.int64)
    if case["prefix"]:
        front = case["prefix"] - (torch.arange(S) * 5) % max(1, case["prefix"] // 2)
    front = torch.minimum(front.repeat_interleave(H), lens)[:, None]
    seen = torch.where(front > at, front, at + 1 - first + torch.minimum(front, first))      # the union of two ranges
    rows = torch.where(front > first[:, :1], lens[:, None], lens[:, None] - first[:, :1] + front)
    return {"bytes": int(rows.sum()) * held + S * n * H * G * (4 * d + 4), "flops": 4 * int(seen.sum()) * G * d}


# ---- in 64 bits, from the definitions -----------------------------------------------------------------------------------------------------

def _exact_rows(s, table, u, row):
    """Those rows of unit u, byte by byte: K, V fp64."""
    d, nb, C = s["d"], s["d"] // 32, _chunk(s["d"])
    size = s["pool"].shape[1]
    flat = s["pool"].view(-1)
    u, row = (u if torch.is_tensor(u) else torch.full_like(row, u))[:, None], row[:, None]
    dim = torch.arange(d, device=flat.device)[None, :]
    page = table[u, row // ROWS].long() * size
    r = row % ROWS
    if s["fmt"] == "16bit":
        words = flat.view(s["dtype"])
        at = page // 2 + r * d + dim
        return words[at].double(), words[at + ROWS * d].double()
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device=flat.device)

    def value(code_at, scale_at):
        code = (flat[code_at] >> (4 * (dim % 2)).to(torch.uint8)) & 15
        return grid[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).double()) * 2.0 ** (flat[scale_at].double() - 127.0)

    block = dim // 32
    k = value(page + r * (d // 2) + dim // 2, page + ROWS * d + block * 64 + r % 16 * 4 + r // 16)
    quad, chunk = r // 4, dim // C
    v = value(page + ROWS * d // 2 + ((quad * (d // C) + chunk) * 4 + r % 4) * (C // 2) + dim % C // 2,
              page + ROWS * d + 2 * d + ((quad % 4 * nb + block) * 4 + r // 16) * 4 + r % 4)
    return k, v


def _exact_beam(s):
    best = torch.full((s["P"], s["n_out"]), -math.inf, dtype=torch.float64, device="cuda")
    for p in range(s["P"]):
        some = []
        for b in range(s["B"]):
            value = s["scores"][p, b].double() + torch.log_softmax(s["logits"][p, b].double(), -1)
            some.append(value[torch.isfinite(value)])
        top = torch.cat(some)
        top = torch.topk(top, min(s["n_out"], top.numel())).values
        best[p, :top.numel()] = top
    return dict(scores=best, beams=None, tokens=None)


def exact(case, seed):
    s = prepare(case, seed)
    if s["path"] == "beam":
        return _exact_beam(s)
    S, H, d = s["S"], s["H"], s["d"]
    if s["path"] in ("copy", "compact"):
        table, parts = s["old_table"] if s["path"] == "compact" else None, []
        if table is None:                                  # the rows of the pages that are copied, found by where they are copied to
            back = torch.zeros(s["pool"].shape[0], dtype=torch.int32, device="cuda")
            back[s["dst"].long()] = s["src"]
            table = torch.where(s["table"] >= 0, back[s["table"].clamp(min=0).long()], -1)
        unit = torch.repeat_interleave(s["head_off"][1:] - s["head_off"][:-1])
        row = s["kept"].long() if s["path"] == "compact" else torch.arange(s["rows"], device="cuda") - s["head_off"][unit]
        for i in range(0, s["rows"], 1 << 18):
            parts.append(_exact_rows(s, table, unit[i:i + (1 << 18)], row[i:i + (1 << 18)]))
        return dict(k=torch.cat([a for a, _ in parts]), v=torch.cat([b for _, b in parts]))
    n, Hq, G = s["n"], s["Hq"], s["Hq"] // H
    attn = torch.zeros(S, n, Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((S, n, Hq), -math.inf, dtype=torch.float64, device="cuda")
    lens = s["lens"].tolist()
    front = [0] * S if s["prefix"] is None else s["prefix"].tolist()
    for u in range(S * H):
        seq, h = divmod(u, H)
        i = torch.arange(lens[u], device="cuda")
        K, V = _exact_rows(s, s["table"], u, i)
        t = torch.arange(n, device="cuda")
        r = (lens[u] - n + t)[:, None]
        seen = (i <= r) & (i > r - s["window"]) if s["window"] else i <= r
        seen = (seen | (i < front[seq])) & (r >= 0)
        for g in range(G):
            z = (s["q"][seq, :, h * G + g].double() @ K.T) * s["scale"]
            if s["cap"]:
                z = s["cap"] * torch.tanh(z / s["cap"])
            if s["slopes"] is not None:
                z -= s["slopes"][h * G + g].double() * (r - i).abs()
            z.masked_fill_(~seen, -math.inf)
            lse[seq, :, h * G + g] = torch.logsumexp(z, -1)
            attn[seq, :, h * G + g] = torch.nan_to_num(torch.softmax(z, -1)) @ V
    return dict(attn=attn, lse=lse)
