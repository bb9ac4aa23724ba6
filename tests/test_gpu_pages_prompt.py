"""Attention of prompts' chunks and single tokens over pages, with rules for the logits, on the GPU against its definition in 64 bits.

Bars, for every number by itself.  A weight is rounded to the rows' type for its product with a value, off by u = half a step of it, so that an output is off by
u sum_i w_i |v_i| at most for normalised weights w; fp16 rows of 4-bit pages: two pieces of bf16, 2^-16.  The output is rounded to the rows' type: u |out|, or half of the smallest
step for fp16's small ones.  Logits carry some 1e-6 from sums, scales, caps and distances in fp32: 1e-5 max|v| as for single tokens' attention, and as much of lse.
"""
import numpy as np
import pytest
import torch

from oracle import pages as op
import paper_2605_26678_amd as nkv
from pages_util import Cache, from_bits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [("bf16", "fp4"), ("fp16", "fp4"), ("bf16", "16bit"), ("fp16", "16bit")]
HEAD_DIMS = [64, 96, 128, 192, 256]
EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 700]


def oracle(q, c, Hq, scale, cap=0.0, window=0, slopes=None, prefix=None):
    """(out, lse, sum of weights times |values|), fp64; rows whose value is not finite make NaN of what sees them."""
    S, n, _, d = q.shape
    H, G = c.H, Hq // c.H
    out, lse, size = np.zeros((S, n, Hq, d)), np.full((S, n, Hq), -np.inf), np.zeros((S, n, Hq, d))
    for u in range(S * H):
        s, h = divmod(u, H)
        length = min(max(int(c.lens[u]), 0), 64 * c.table.shape[1])
        K, V, there = np.zeros((length, d)), np.zeros((length, d)), np.zeros(length, bool)
        for j in range((length + 63) // 64):
            p = int(c.table[u, j])
            if 0 <= p < c.pool.shape[0]:
                k, v = op.read_rows(c.pool[p], d, c.fp4, from_bits(c.torch_dtype))
                m = min(64, length - 64 * j)
                K[64 * j:64 * j + m], V[64 * j:64 * j + m], there[64 * j:64 * j + m] = k[:m], v[:m], True
        i = np.arange(length)
        r = length - n + np.arange(n)[:, None]
        see = i <= r
        if window:
            see &= i > r - window
        if prefix is not None:
            see |= i < int(prefix[s])
        see &= (r >= 0) & there
        for g in range(G):
            with np.errstate(all="ignore"):
                z = scale * (q[s, :, h * G + g] @ np.where(np.isfinite(K), K, 0.0).T)
                if cap:
                    z = cap * np.tanh(z / cap)
                if slopes is not None:
                    z = z - float(slopes[h * G + g]) * np.abs(r - i)
                z = np.where(see, z, -np.inf)
            some = see.any(1)
            z = z[some]
            if not z.size:
                continue
            top = z.max(1, keepdims=True)
            e = np.where(see[some], np.exp(z - top), 0.0)
            total = e.sum(1, keepdims=True)
            bad = ~np.isfinite(V).all(1)
            W = np.where(np.isfinite(V), V, 0.0)
            out[s, some, h * G + g] = (e / total) @ W
            size[s, some, h * G + g] = (e / total) @ np.abs(W)
            lse[s, some, h * G + g] = top[:, 0] + np.log(total[:, 0])
            poisoned = (see[some] & (bad | ~np.isfinite(K).all(1))).any(1)
            out[s, np.flatnonzero(some)[poisoned], h * G + g] = np.nan
    return out, lse, size


def attend(c, q, Hq, scale, stream=None, want_lse=True, **rules):
    """A call with room to spare around out and lse, and none around the scratch, which holds NaN before."""
    pages = c.on(DEV)
    n = q.shape[1]
    need = nkv.pages_prompt_workspace_bytes(pages, Hq, n)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((c.S * n * Hq * c.d + 128,), -77.0, dtype=c.torch_dtype, device=DEV)
    lse = torch.full((c.S * n * Hq + 128,), -77.0, device=DEV)
    o, l = out[64:-64].view(c.S, n, Hq, c.d), lse[64:-64].view(c.S, n, Hq)
    made = nkv.LogitRules(rules.get("cap", 0.0), rules.get("window", 0), *[None if rules.get(k) is None else torch.as_tensor(rules[k]).to(DEV) for k in ("slopes", "prefix")])
    torch.cuda.synchronize()
    nkv.pages_prompt_attention(q.to(DEV), pages, Hq, n, scale, o, l if want_lse else None, ws[:need], rules=made if rules else None, stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all()), "written behind the scratch"
    for x in (out[:64], out[-64:], lse[:64], lse[-64:]):
        assert bool((x == -77.0).all()), "written beside the outputs"
    assert torch.equal(c.d_pool.cpu(), torch.from_numpy(c.pool)) and torch.equal(c.d_lens.cpu(), torch.from_numpy(c.lens))
    return o, l


def check(c, q, Hq, scale, what, **rules):
    o, l = attend(c, q, Hq, scale, **rules)
    want, want_lse, size = oracle(q.double().numpy(), c, Hq, scale, **rules)
    got, got_lse = o.cpu().double().numpy(), l.cpu().double().numpy()
    nan = np.isnan(want).any(-1)
    assert not np.isfinite(got[nan]).all(-1).any(), f"{what}: a row of NaN left no trace"
    assert np.isfinite(got[~nan]).all(), f"{what}: not finite"
    u = torch.finfo(c.torch_dtype).eps / 2
    weight = 2.0 ** -16 if c.fp4 and c.torch_dtype == torch.float16 else u
    tiny = float(torch.finfo(c.torch_dtype).smallest_normal) * u
    bar = weight * size + u * np.abs(want) + tiny + 1e-5 * max(1.0, np.nanmax(size, initial=0.0))
    off = (np.abs(got - want) / bar)[~nan]
    assert off.size == 0 or off.max() <= 1.0, f"{what}: {off.max():.2f} times what roundings leave"
    fin = np.isfinite(want_lse) & ~nan
    assert np.array_equal(np.isneginf(got_lse[~nan]), np.isneginf(want_lse[~nan])), what
    e = np.abs(got_lse[fin] - want_lse[fin]) / np.maximum(1.0, np.abs(want_lse[fin]))
    assert e.size == 0 or e.max() <= 1e-5, f"{what}: lse off by {e.max():.3e}"
    return o, l


def queries(c, n, Hq, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(c.S, n, Hq, c.d, generator=g)).to(c.torch_dtype)


def slopes_of(Hq):
    return (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)


# pages of a unit's row of the table, by which calls of few columns go with one kernel or the other
WIDTHS = [None, 40]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("d", HEAD_DIMS)
def test_lengths(d, dtype, fmt, width):
    c = Cache(4, 4, d, dtype, fmt, EDGES, width=width, seed=d, rows=1.0)
    for n, G in ((1, 1), (1, 8), (2, 16), (5, 3), (40, 1), (70, 4)) if width is None else ((1, 1), (1, 8), (2, 16), (5, 3)):
        check(c, queries(c, n, 4 * G, n), 4 * G, 1 / np.sqrt(d), f"{n} tokens of {G} heads")


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_the_largest_window_and_tokens_in_front_of_the_first_row(dtype, fmt, width):
    c = Cache(4, 4, 64, dtype, fmt, EDGES, width=width, seed=2, rows=1.0)
    for n, G in ((300, 1), (7, 2)):
        q = queries(c, n, 4 * G, n)
        for window in ((1 << 31) - 1, 1 << 30, 3):
            check(c, q, 4 * G, 0.125, f"{n} tokens, window {window}", window=window, prefix=np.array([0, 40, 1 << 30, 20], np.int32))


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("d", HEAD_DIMS)
@pytest.mark.parametrize("width", WIDTHS)
def test_rules(d, dtype, fmt, width):
    c = Cache(3, 2, d, dtype, fmt, [700, 333, 130, 64, 40, 3], width=width, seed=d + 1, rows=1.0)
    slopes = slopes_of(6)
    for n in (1, 4, 90) if width is None else (1, 4):
        q = queries(c, n, 6, n, 2.0)
        for rules in (dict(cap=1.5), dict(cap=6.0), dict(cap=30.0), dict(cap=100.0), dict(window=1), dict(window=70), dict(prefix=np.array([100, 0, 500], np.int32)), dict(slopes=slopes),
                      dict(window=37, prefix=np.array([65, 129, 2], np.int32)), dict(cap=5.0, window=150, slopes=slopes, prefix=np.array([4, -3, 1 << 30], np.int32))):
            check(c, q, 6, 1 / np.sqrt(d), f"{n} tokens, {rules}", **rules)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_windows_and_prefixes_at_page_borders(dtype, fmt, width):
    c = Cache(2, 1, 64, dtype, fmt, [640, 577], width=width, seed=3, rows=1.0)
    for n in (1, 3, 200) if width is None else (1, 3):
        q = queries(c, n, 2, n)
        for window in (1, 63, 64, 65, 128, 129, 640, 1 << 30):
            for prefix in (None, np.array([64, 1], np.int32), np.array([63, 65], np.int32), np.array([639, 577], np.int32)):
                check(c, q, 2, 0.125, f"{n} tokens, window {window}, prefix {prefix}", window=window, **({} if prefix is None else dict(prefix=prefix)))


@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_long(dtype, fmt):
    # rows shared out among workgroups, and several tiles of columns
    c = Cache(1, 2, 128, dtype, fmt, [5000, 4321], seed=5, rows=1.0)
    for n, G in ((1, 1), (1, 8), (3, 5), (16, 1), (17, 1), (4, 8), (33, 1), (150, 4)):
        check(c, queries(c, n, 2 * G, n), 2 * G, 1 / np.sqrt(128), f"{n} tokens of {G} heads")
    check(c, queries(c, 17, 4, 4), 4, 0.1, "rules", cap=20.0, window=1000, prefix=np.array([700], np.int32), slopes=slopes_of(4))
    check(c, queries(c, 1, 4, 4), 4, 0.1, "rules", cap=20.0, window=1000, prefix=np.array([700], np.int32), slopes=slopes_of(4))


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("n", [1, 3, 90])
def test_pages_that_are_none_and_wide_tables(n, dtype, fmt):
    c = Cache(2, 2, 128, dtype, fmt, [700, 300, 64, 129], width=40, seed=6, rows=1.0)
    c.table[0, 2], c.table[0, 10], c.table[1, 0], c.table[2, 0] = -1, c.pool.shape[0], -5, 1 << 30
    check(c, queries(c, n, 8, 1), 8, 0.1, "holes")
    check(c, queries(c, n, 8, 1), 8, 0.1, "holes", window=100, prefix=np.array([150, 10], np.int32))
    c.lens[:] = [1 << 30, -7, 64 * 40, 5]                                  # beyond the table, negative
    check(c, queries(c, n, 8, 1), 8, 0.1, "lengths")


@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("d", HEAD_DIMS)
def test_short_caches(d, dtype, fmt):
    """Up to 16 columns of units of a few pages, in one launch."""
    for lens in ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 120, 127, 128], [5, 500, 64, 449, 448, 1, 0, 129] * 2):
        c = Cache(4, 4, d, dtype, fmt, lens, seed=d, rows=1.0)
        for n, G in ((1, 1), (1, 16), (2, 8), (3, 5), (16, 1)):
            q = queries(c, n, 4 * G, n)
            check(c, q, 4 * G, 1 / np.sqrt(d), f"{n} tokens of {G} heads")
            check(c, q, 4 * G, 0.3, f"{n} tokens of {G} heads, rules", cap=20.0, window=70, slopes=slopes_of(4 * G), prefix=np.array([0, 3, 100, 1000], np.int32))


@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_short_windows_of_long_caches(dtype, fmt):
    """One launch by the window, without a prefix or with many units; prefixes of any number of pages."""
    c = Cache(2, 2, 128, dtype, fmt, [1500, 2999, 3, 1111], width=200, seed=3, rows=1.0)
    for n, window, prefix in ((1, 1, [0, 0]), (1, 64, None), (2, 65, None), (3, 200, [1000, 1400]), (1, 130, [5000, -3]), (1, 700, None)):
        check(c, queries(c, n, 8, n), 8, 0.1, f"{n} tokens, window {window}, prefix {prefix}", window=window, prefix=None if prefix is None else np.array(prefix, np.int32), cap=30.0)
    c = Cache(64, 4, 64, dtype, fmt, [65 + u * 7 % 400 for u in range(256)], width=24, seed=4, rows=1.0)
    check(c, queries(c, 2, 4, 2), 4, 0.1, "many units", window=40, prefix=np.arange(-3, 61, dtype=np.int32) * 5, slopes=slopes_of(4))


def _plant(c, u, row, value, key=False, dim=5):
    """Infinity or NaN into a row of V (or K)."""
    page = c.pool[c.table[u, row // 64]]
    if c.fp4:
        _, _, ks, vs = op.places(c.d)
        page[(ks if key else vs)[row % 64, dim // 32]] = 255
        return
    w = page.view(np.uint16).reshape(2, 64, c.d)
    w[0 if key else 1, row % 64, dim] = torch.tensor(value, dtype=c.torch_dtype).view(torch.int16).item() & 0xffff


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_rows_that_are_not_seen_hold_anything(dtype, fmt, value, width):
    for d in (64, 128, 256):
        for n, planted in ((1, [3, 100]), (3, [3, 150, 297, 299]), (90, [3, 70, 215, 260, 299]), (90, [5, 298])):
            if width and n > 3:
                continue
            for key in (False, True):                                     # (an infinite key is a logit of either infinity: keys of NaN)
                c = Cache(1, 1, d, dtype, fmt, [300], width=width, seed=d, rows=1.0)
                for row in planted:
                    _plant(c, 0, row, float("nan") if key else value, key=key)
                q = queries(c, n, 3, n)
                # only what sees none of the rows is finite, and right
                check(c, q, 3, 0.1, f"{n} tokens", window=60)
                check(c, q, 3, 0.1, f"{n} tokens", window=2)


def _enlarge(c, u, row):
    """Keys of a row 2^6 times as large: finite, and far beyond any cap."""
    page = c.pool[c.table[u, row // 64]]
    if c.fp4:
        page[op.places(c.d)[2][row % 64]] += 6
    else:
        k = page.view(np.uint16).reshape(2, 64, c.d)[0, row % 64]
        k[:] = (torch.from_numpy(k.view(np.int16).copy()).view(c.torch_dtype) * 64).view(torch.int16).numpy().view(np.uint16)


@pytest.mark.parametrize("cap", [0.0, 5.0, 20.0, 50.0, 100.0])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_rows_that_are_not_seen_leave_every_bit(dtype, fmt, width, cap):
    """Of other tokens' rows, and of those behind the last one, no part has any: outputs and log sums of the tokens that do not see them are the same to the bit."""
    for d in (64, 128, 192):
        for n, G, scale in ((1, 2, 0.1), (3, 2, 0.1), (90, 3, 0.1), (90, 3, 0.9)):
            if width and n > 3:
                continue
            c = Cache(1, 1, d, dtype, fmt, [300], width=width, seed=d, rows=1.0)
            q = queries(c, n, G, n)
            rules = dict(cap=cap, window=60, prefix=np.array([7], np.int32))
            o, l = (x.clone() for x in attend(c, q, G, scale, **rules))
            # in front of all windows or of some, behind the last one, in the middle of the tokens, the last one
            rows = [20, 230, 303] + ([299 - n // 2, 299] if n > 1 else [])
            for row in rows:
                _enlarge(c, 0, row)
            o2, l2 = attend(c, q, G, scale, **rules)
            r = 300 - n + np.arange(n)
            blind = np.ones(n, bool)
            for row in rows:
                blind &= ~((row <= r) & (row > r - 60))
            assert blind.all() if n == 1 else 0 < blind.sum() < n
            assert torch.equal(o[:, blind], o2[:, blind]) and torch.equal(l[:, blind], l2[:, blind]), f"{d}, {n}, {scale}"


@pytest.mark.parametrize("d,scale,cap", [(128, 128 ** -0.5, 100.0), (128, 1 / 128, 30.0), (256, 1 / 16, 70.0), (64, 0.125, 2000.0), (192, 0.01, 64.0), (128, 0.1, 2e4)])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_rows_that_are_not_seen_leave_every_bit_under_wide_caps(dtype, fmt, width, d, scale, cap):
    """Caps of a thousand scales and more, with one polynomial for small logits, and none: how a column's logits are capped does not go by its neighbours'."""
    for n, G in ((2, 3), (3, 2), (90, 3), (90, 1)):
        if width and n > 3:
            continue
        c = Cache(1, 1, d, dtype, fmt, [300], width=width, seed=d, rows=1.0)
        q = queries(c, n, G, n)
        rules = dict(cap=cap, window=60, prefix=np.array([7], np.int32))
        o, l = (x.clone() for x in check(c, q, G, scale, f"{n} tokens", **rules))
        for _ in range(2):                                                 # twice: beyond what any polynomial takes
            _enlarge(c, 0, 300 - n // 2)
        o2, l2 = attend(c, q, G, scale, **rules)
        blind = 300 - n + np.arange(n) < 300 - n // 2
        assert 0 < blind.sum() < n
        assert torch.equal(o[:, blind], o2[:, blind]) and torch.equal(l[:, blind], l2[:, blind]), f"{n} tokens of {G} heads"


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_far_logits_of_other_columns_leave_every_bit(dtype, fmt, width, d):
    """The last token's logits are beyond 2^24 by its own row, which no other sees."""
    for n, G in ((2, 8), (3, 5), (90, 3)):
        if width and n > 3:
            continue
        for rules in (dict(), dict(window=200), dict(slopes=slopes_of(G))):
            c = Cache(1, 1, d, dtype, fmt, [300], width=width, seed=d, rows=1.0)
            q = queries(c, n, G, n)
            q[:, -1] *= 8192
            q[:, -1, 1] = -q[:, -1, 0]                                     # (the row's logit is positive of one of the two)
            o, l = (x.clone() for x in attend(c, q, G, 0.3, **rules))
            assert float(l[:, -1].abs().max()) < 2.0 ** 20
            for _ in range(2):
                _enlarge(c, 0, 299)
            o2, l2 = attend(c, q, G, 0.3, **rules)
            assert float(l2[:, -1].abs().max()) > 2.0 ** 24
            assert torch.equal(o[:, :-1], o2[:, :-1]) and torch.equal(l[:, :-1], l2[:, :-1]), f"{n} tokens of {G} heads, {list(rules)}"


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype,fmt", KINDS)
@pytest.mark.parametrize("n", [1, 2, 40])
def test_scales(n, dtype, fmt, width):
    c = Cache(1, 2, 64, dtype, fmt, [200, 77], width=width, seed=8, rows=1.0)
    q = queries(c, n, 4, 2)
    for scale in (-0.2, 0.0, 1e-40, -1e-46, 3.0):
        check(c, q, 4, scale, f"scale {scale}")
    for rules in (dict(cap=3.0), dict(slopes=slopes_of(4)), dict(cap=3.0, slopes=-slopes_of(4))):
        for scale in (-0.2, 0.0, 3.0):
            check(c, q, 4, scale, f"scale {scale}, {rules}", **rules)
    check(c, q, 4, 0.5, "a cap that nothing comes near", cap=1e6)
    check(c, q, 4, 0.5, "a small cap", cap=1e-3)
    for cap in (0.2, 2.0, 5.0, 20.0, 63.0, 65.0, 300.0):
        for scale in (0.02, 0.3, 5.0, 40.0):
            check(c, q, 4, scale, f"scale {scale}, cap {cap}", cap=cap)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dtype,fmt", KINDS)
def test_far_logits(n, dtype, fmt, width):
    """Logits of 2^26 and more: one row has all the weight, or, where their places are wider than their distance, some."""
    c = Cache(1, 1, 64, dtype, fmt, [150], width=width, seed=9, rows=1.0)
    for scale in (1e7, -1e7, 1e30):
        o, l = attend(c, queries(c, n, 2, 3), 2, scale)
        assert bool(o.isfinite().all()) and bool(l.isfinite().all())
    # one row along the query: the output is its value
    if fmt == "16bit":
        w = c.pool[c.table[0, 1]].view(np.uint16).reshape(2, 64, 64)
        q = queries(c, n, 2, 3)
        q[:] = q[:, :1, :1]
        w[0, 7] = (q[0, 0, 0] * 8).view(torch.int16).numpy().view(np.uint16)
        o, l = attend(c, q, 2, 1e8)
        value = torch.from_numpy(w[1, 7].view(np.int16).copy()).view(c.torch_dtype)
        assert torch.equal(o.cpu(), value.expand_as(o.cpu()))


def test_calls_are_deterministic_on_streams_and_in_graphs():
    side = torch.cuda.Stream()
    for n, G, lens in ((1, 4, [5000, 700]), (2, 3, [900, 64]), (1, 2, [200, 100]), (130, 4, [3000, 1000])):
        c = Cache(1, 2, 128, "bf16", "fp4", lens, seed=n, rows=1.0)
        Hq, slopes = 2 * G, slopes_of(2 * G)
        q = queries(c, n, Hq, 7)
        kw = dict(cap=30.0, window=2000, slopes=slopes, prefix=np.array([10], np.int32))
        want = attend(c, q, Hq, 0.1, **kw)
        side.wait_stream(torch.cuda.current_stream())
        for stream in (None, side):
            for a, b in zip(attend(c, q, Hq, 0.1, stream=stream, **kw), want):
                assert torch.equal(a, b)
        assert torch.equal(attend(c, q, Hq, 0.1, want_lse=False, **kw)[0], want[0])
        # lengths, queries and tables are read at every replay; two graphs share a scratch
        pages = c.on(DEV)
        d_q, rules = q.to(DEV), nkv.LogitRules(30.0, 2000, torch.from_numpy(slopes).to(DEV), torch.tensor([10], dtype=torch.int32, device=DEV))
        ws = torch.empty(max(256, nkv.pages_prompt_workspace_bytes(pages, Hq, n)), dtype=torch.uint8, device=DEV)
        out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                nkv.pages_prompt_attention(d_q, pages, Hq, n, 0.1, out, lse, ws, rules=rules)
            graphs.append(graph)
        for i in range(4):
            d_q.copy_(queries(c, n, Hq, 20 + i))
            c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32) - 13 * i)
            out.fill_(float("nan"))
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            o, l = torch.zeros_like(out), torch.zeros_like(lse)
            nkv.pages_prompt_attention(d_q, pages, Hq, n, 0.1, o, l, ws, rules=rules)
            torch.cuda.synchronize()
            assert torch.equal(o, out) and torch.equal(l, lse)


def test_agrees_with_single_tokens_attention():
    """A prompt's chunk without rules is what the other call computes token by token."""
    for dtype, fmt in KINDS:
        c = Cache(2, 2, 128, dtype, fmt, [500, 130, 64, 333], seed=11, rows=1.0)
        q = queries(c, 33, 8, 1)
        o, l = attend(c, q, 8, 0.1)
        pages = c.on(DEV)
        out, lse = torch.empty(2, 33, 8, 128, device=DEV), torch.empty(2, 33, 8, device=DEV)
        ws = torch.empty(nkv.pages_workspace_bytes(pages, 8, 33), dtype=torch.uint8, device=DEV)
        nkv.pages_attention(q.to(DEV), pages, 8, 33, 0.1, out, lse, ws)
        # (a weight's rounding, and the output's)
        assert (o.float() - out).abs().max() <= 2 * torch.finfo(c.torch_dtype).eps / 2 * 6.0 + 1e-5
        assert torch.allclose(l, lse, rtol=1e-5, atol=1e-5)
