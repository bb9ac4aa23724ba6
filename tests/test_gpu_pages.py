"""The paged cache on the GPU against oracle/pages.py.

Bars.  What is written to pages, read from them, and rotated is compared bit for bit: a rotation in 64 bits rounded to 32 is the same
number whatever the order of its operations, and a code is the nearest one of the value so rounded.  Attention: |out - oracle| <=
1e-5 max(1, max|V|), with 6 for max|V|, |lse - oracle| <= 1e-5 max(1, |lse|), as for attention over packed rows: the products are exact, logits of a few tens
at most carry some 1e-6 from their sums in fp32, and the output is a convex combination of value rows.  At logits of a few the bar is 2e-6 of the
largest value that is there (pages_util.attention_bar), which a lost piece of the weights leaves.
"""
import numpy as np
import pytest
import torch

from oracle import pages as op
import nkv_inputs
import paper_2605_26678_amd as nkv
from pages_util import Cache, DTYPES, attention_bar, from_bits, to_bits, values_of
from parity_util import shape_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 1e-5


def _f64(t):
    return t.detach().cpu().double().numpy()


def _attend(c, q, scale, n, Hq, want_lse=True, stream=None):
    """A call with room to spare around out and lse, and none around the scratch, which holds NaN before."""
    pages = c.on(DEV)
    need = nkv.pages_workspace_bytes(pages, Hq, n)
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device=DEV)
    out = torch.full((c.S * n * Hq * c.d + 128,), float("nan"), device=DEV)
    lse = torch.full((c.S * n * Hq + 128,), float("nan"), device=DEV)
    o, l = out[64:-64].view(c.S, n, Hq, c.d), lse[64:-64].view(c.S, n, Hq)
    torch.cuda.synchronize()
    nkv.pages_attention(q.to(DEV), pages, Hq, n, scale, o, l if want_lse else None, ws[:need], stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 255).all()), "written behind the scratch"
    for x in (out[:64], out[-64:], lse[:64], lse[-64:]):
        assert bool(x.isnan().all()), "written beside the outputs"
    assert torch.equal(c.d_pool.cpu(), torch.from_numpy(c.pool)) and torch.equal(c.d_lens.cpu(), torch.from_numpy(c.lens))
    return o, l


def _check(c, q, o, l, scale, what, n):
    want, want_lse = op.attention(_f64(q), c.pool, c.table, c.lens, c.H, scale, c.d, c.fp4, from_bits(c.torch_dtype))
    vmax = 6.0 if c.fp4 else 6.0                           # codes of up to 6 * 2^-1, rows of a few standard deviations
    assert np.isfinite(_f64(o)).all(), what
    err = np.abs(_f64(o) - want).max()
    assert err <= TOL * max(1.0, vmax), f"{what}: out off by {err:.3e}"
    if l is not None:
        assert np.array_equal(np.isneginf(_f64(l)), np.isneginf(want_lse)), what
        fin = np.isfinite(want_lse)
        e2 = np.abs(_f64(l)[fin] - want_lse[fin]) / np.maximum(1.0, np.abs(want_lse[fin]))
        assert e2.size == 0 or e2.max() <= TOL, f"{what}: lse off by {e2.max():.3e}"


def _queries(c, n, Hq, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(c.S, n, Hq, c.d, generator=g).to(c.torch_dtype)


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 700]


# ---- rows in and out ----

def _append_case(c, n, Hq, rot, halves, seed, positions=None, fused=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(c.S, n, Hq + 2 * c.H, c.d, generator=g) * torch.exp(torch.randn(c.S, n, Hq + 2 * c.H, 1, generator=g))
    x = x.to(c.torch_dtype)
    rope = nkv.rope_table(60, rot, device="cpu") if rot else None
    if positions is None:
        positions = torch.randint(0, 60, (c.S, n), generator=g, dtype=torch.int32)
    if not fused:                                          # heads outside of tokens, and a hole between sequences
        wide = torch.zeros(c.S, Hq + 2 * c.H, n + 1, c.d, dtype=x.dtype)
        wide[:, :, :n] = x.transpose(1, 2)
        x = wide[:, :, :n].transpose(1, 2)
    return x, rope, positions


def _append_oracle(c, x, rope, positions, n, Hq, rot, halves):
    """The pool after the call, and q_out (NaN where nothing is written)."""
    pool, bits = c.pool.copy(), to_bits(c.torch_dtype)
    f = _f64(x)
    q, k, v = f[:, :, :Hq], f[:, :, Hq:Hq + c.H], f[:, :, Hq + c.H:]
    pos = positions.numpy()
    if rot:
        q, k = (op.rotate(t, pos, rope.numpy(), halves) for t in (q, k))
    q_out = np.full(q.shape, np.nan)
    for s in range(c.S):
        for t in range(n):
            if rot and not 0 <= pos[s, t] < rope.shape[0] or pos[s, t] < 0:
                continue
            q_out[s, t] = from_bits(c.torch_dtype)(bits(q[s, t]).reshape(-1)).reshape(Hq, c.d)
            for h in range(c.H):
                u = s * c.H + h
                row = min(max(int(c.lens[u]), 0), 64 * c.width) - n + t
                if row < 0:
                    continue
                p = int(c.table[u, row // 64])
                if 0 <= p < pool.shape[0]:
                    op.write_row(pool[p], row % 64, True, k[s, t, h], c.fp4, bits)
                    op.write_row(pool[p], row % 64, False, v[s, t, h], c.fp4, bits)
    return pool, q_out


def _run_append(c, x, rope, positions, n, Hq, rot, halves, give_positions=True):
    pages = c.on(DEV)
    d = x.to(DEV) if x.is_contiguous() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=DEV).copy_(x)
    q_out = torch.full((c.S, n, Hq, c.d), float("nan"), dtype=x.dtype, device=DEV) if Hq else None
    torch.cuda.synchronize()
    nkv.pages_append(d[:, :, Hq:Hq + c.H], d[:, :, Hq + c.H:], pages, positions=positions.to(DEV) if give_positions else None,
                     rope=rope.to(DEV) if rot else None, rope_style=nkv.ROPE_HALVES if halves else nkv.ROPE_PAIRS,
                     q=d[:, :, :Hq] if Hq else None, q_out=q_out)
    torch.cuda.synchronize()
    return c.d_pool.cpu().numpy(), q_out


@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("dtype,halves,part", [("bf16", True, 1), ("bf16", False, 1), ("fp16", True, 2), ("fp16", False, 2), ("bf16", True, 0)])
def test_append_writes_the_oracles_bytes(d, fmt, dtype, halves, part):
    rot = d // part if part else 0
    n, Hq = 5, 4
    c = Cache(2, 2, d, dtype, fmt, [5, 64, 67, 131], rows=1.0, seed=d)
    x, rope, positions = _append_case(c, n, Hq, rot, halves, 7 * d, fused=halves)
    want, want_q = _append_oracle(c, x, rope, positions, n, Hq, rot, halves)
    got, q_out = _run_append(c, x, rope, positions, n, Hq, rot, halves, give_positions=bool(rot))
    assert np.array_equal(got, want), f"{(got != want).sum()} bytes differ"
    assert np.array_equal(_f64(q_out), want_q)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_append_leaves_out_padding_foreign_positions_and_pages_that_are_none(fmt):
    """Leading tokens of negative positions, positions behind the table, rows in front of row 0, table entries outside the pool, lengths
    beyond the table's row and below zero."""
    n, Hq = 6, 2
    c = Cache(4, 2, 64, "bf16", fmt, [70, 6, 3, 0, 130, 66, 64, 64], width=3, rows=1.0, seed=5)
    c.table[4, 2], c.table[5, 1] = c.pool.shape[0], -7
    c.lens[6], c.lens[7] = 1000, -3                        # clamped to 192 rows (two pages there are none) and to none
    x, rope, positions = _append_case(c, n, Hq, 64, True, 3)
    positions[0, :3] = -1
    positions[1, 2] = 60
    want, want_q = _append_oracle(c, x, rope, positions, n, Hq, 64, True)
    got, q_out = _run_append(c, x, rope, positions, n, Hq, 64, True)
    assert np.array_equal(got, want)
    assert np.array_equal(_f64(q_out), want_q, equal_nan=True)


@pytest.mark.parametrize("S,n,H,G,d,rot,halves,dtype,fmt", [
    (2, 3, 32, 1, 96, 48, False, "fp16", "fp4"),          # 96 rows, 21 at a time: five workgroups a token, the last one partly filled
    (2, 3, 8, 4, 256, 256, False, "bf16", "16bit"),       # 48 rows, 8 at a time: six workgroups a token
    (3, 1, 8, 4, 256, 256, True, "bf16", "fp4"),          # 16 at a time: three
    (1, 700, 8, 4, 256, 128, False, "bf16", "fp4"),       # two workgroups a token, three rounds each
    (1, 900, 32, 1, 96, 96, True, "bf16", "16bit"),       # two workgroups, 42 rows at a time: the second one's last round is partly filled
    (3, 701, 8, 4, 128, 128, True, "bf16", "fp4"),        # more than 2048 tokens: one workgroup each, 32 rows and 16 more
    (3, 701, 8, 4, 128, 32, True, "fp16", "16bit"),
    (1, 2113, 32, 2, 64, 16, False, "fp16", "fp4"),
])
def test_append_with_many_heads_and_tokens(S, n, H, G, d, rot, halves, dtype, fmt):
    """A token's rows shared out to several workgroups, and more of them than a workgroup takes at a time: sampled tokens' rows of all heads against the oracle, and
    the rows in front of the new ones as they were."""
    Hq, held = H * G, 37
    c = Cache(S, H, d, dtype, fmt, [held + n] * (S * H), rows=1.0, seed=n)
    x, rope, positions = _append_case(c, n, Hq, rot, halves, 11 * n)
    before = c.pool.copy()
    got, q_out = _run_append(c, x, rope, positions, n, Hq, rot, halves)
    f, q_out = _f64(x), _f64(q_out)
    bits, back = to_bits(c.torch_dtype), from_bits(c.torch_dtype)
    spread = sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n)))
    for s in range(S):
        for t in spread:
            pos = positions[s:s + 1, t:t + 1].numpy()
            turned = op.rotate(f[s:s + 1, t:t + 1, :Hq + H], pos, rope.numpy(), halves)[0, 0]
            assert np.array_equal(q_out[s, t], back(bits(turned[:Hq]).reshape(-1)).reshape(Hq, d)), (s, t)
            for h in range(H):
                at, row = c.table[s * H + h, (held + t) // 64], (held + t) % 64
                want = got[at].copy()
                op.write_row(want, row, True, turned[Hq + h], c.fp4, bits)
                op.write_row(want, row, False, f[s, t, Hq + H + h], c.fp4, bits)
                assert np.array_equal(want, got[at]), (s, t, h)
        for h in range(H):
            for key_value in zip(*(op.read_rows(p[c.table[s * H + h, 0]], d, c.fp4, back) for p in (before, got))):
                assert np.array_equal(key_value[0][:held], key_value[1][:held])
    # no row was left out: none of the new ones is what was there
    for u in range(S * H):
        for j in range((held + n + 63) // 64):
            old, new = (np.concatenate(op.read_rows(p[c.table[u, j]], d, c.fp4, back), -1) for p in (before, got))
            lo, hi = max(held - 64 * j, 0), min(held + n - 64 * j, 64)
            assert (old[lo:hi] != new[lo:hi]).any(-1).all(), (u, j)


@pytest.mark.parametrize("d,rot", [(128, 32), (128, 16), (64, 16), (96, 32), (192, 64), (256, 48)])
@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("halves", [True, False])
def test_append_rotates_a_part_of_a_row(d, rot, fmt, halves):
    n, Hq = 4, 4
    c = Cache(2, 2, d, "bf16", fmt, [4, 64, 66, 130], rows=1.0, seed=rot)
    x, rope, positions = _append_case(c, n, Hq, rot, halves, 3 * d + rot)
    want, want_q = _append_oracle(c, x, rope, positions, n, Hq, rot, halves)
    got, q_out = _run_append(c, x, rope, positions, n, Hq, rot, halves)
    assert np.array_equal(got, want), f"{(got != want).sum()} bytes differ"
    assert np.array_equal(_f64(q_out), want_q)


def test_append_without_queries_and_one_token():
    c = Cache(3, 1, 128, "fp16", "fp4", [1, 64, 65], rows=1.0, seed=6)
    x, rope, positions = _append_case(c, 1, 0, 128, True, 8)
    want, _ = _append_oracle(c, x, rope, positions, 1, 0, 128, True)
    got, _ = _run_append(c, x, rope, positions, 1, 0, 128, True)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_4_bit_codes_of_ties_zeros_extremes_and_nan(dtype):
    """Every half-way point, zeros, the smallest and largest values of the type, a NaN and an infinity in a block each."""
    c = Cache(1, 1, 64, dtype, "fp4", [64], seed=9)
    half = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    x = torch.zeros(64, 64)
    for i in range(40):
        scale = 2.0 ** (i - 20 if dtype == "bf16" else i % 20 - 10)
        x[i, :8], x[i, 8:16] = half * scale, -half * scale
        x[i, 32:40] = half * scale * (1 + 2.0 ** -7)
        x[i, 41] = 7.0 * scale
        x[i, 42] = 6.96875 * scale
    top, tiny = torch.finfo(DTYPES[dtype][0]).max, torch.finfo(DTYPES[dtype][0]).tiny
    x[40, :32], x[41, :32], x[42, :32] = top, tiny, tiny / 64
    x[43, 3], x[44, 35], x[45, 63] = float("nan"), float("inf"), -float("inf")
    x[46] = -0.0
    rows = x.to(c.torch_dtype)
    pages = c.on(DEV)
    off = torch.tensor([0, 64], device=DEV)
    nkv.pages_load(rows.to(DEV), rows.flip(0).contiguous().to(DEV), off, 64, pages)
    torch.cuda.synchronize()
    want, f = c.pool.copy(), _f64(rows)
    for r in range(64):
        op.write_row(want[c.table[0, 0]], r, True, f[r], True, None)
        op.write_row(want[c.table[0, 0]], r, False, f[63 - r], True, None)
    assert np.array_equal(c.d_pool.cpu().numpy(), want)
    k, v = torch.empty_like(rows, device=DEV), torch.empty_like(rows, device=DEV)
    nkv.pages_read(k, v, off, 64, pages)
    K, V = op.read_rows(want[c.table[0, 0]], 64, True, None)
    for got, exact in ((k, K), (v, V)):
        as_type = torch.from_numpy(np.clip(exact, -top, top)).to(c.torch_dtype)
        assert torch.equal(got.cpu().nan_to_num(7.0), as_type.nan_to_num(7.0))
        assert torch.equal(got.cpu().isnan(), as_type.isnan())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_every_code_with_every_scale_reads_as_its_value(dtype):
    """Rows of all 16 codes under all 256 scale bytes, as K and as V; values between the type's steps are rounded to nearest, ties to even."""
    c = Cache(1, 1, 64, dtype, "fp4", [256], seed=10)
    codes = np.tile(np.arange(16, dtype=np.uint8), 4)
    k, v, ks, vs = op.places(64)
    for j in range(4):
        page = c.pool[c.table[0, j]]
        for r in range(64):
            for at in (k, v):
                page[at[r, 0::2]] = codes[0::2] | codes[1::2] << 4
            page[ks[r]], page[vs[r]] = 64 * j + r, 255 - (64 * j + r)
    off = torch.tensor([0, 256], device=DEV)
    back = [torch.empty(256, 64, dtype=c.torch_dtype, device=DEV) for _ in range(2)]
    nkv.pages_read(back[0], back[1], off, 256, c.on(DEV))
    top = torch.finfo(c.torch_dtype).max
    for got, scales in zip(back, (np.arange(256), 255 - np.arange(256))):
        exact = op.values(np.tile(codes, (256, 1)), np.repeat(scales[:, None], 2, 1).astype(np.uint8))
        want = torch.from_numpy(np.clip(exact, -top, top)).to(c.torch_dtype)
        assert torch.equal(got.cpu().isnan(), want.isnan())
        assert torch.equal(got.cpu().nan_to_num(7.0)[scales >= 1], want.nan_to_num(7.0)[scales >= 1])   # (0 is no scale that is written)


def _bits(t):
    """A 16-bit tensor's bits, of NaN all the same (and not those of an infinity, which is no largest finite value)."""
    return torch.where(t.isnan(), torch.full_like(t, float("nan")), t).cpu().contiguous().view(torch.int16)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_values_beyond_the_type_read_as_its_largest_finite_one(dtype):
    """All 16 codes under all scale bytes that are written (1 .. 255), as K and as V, compared as bits: no infinity comes out.  The smallest magnitude, 0.5,
    is beyond fp16 from scale byte 144 on."""
    c = Cache(1, 1, 64, dtype, "fp4", [256], seed=30)
    codes = np.tile(np.arange(16, dtype=np.uint8), 4)
    k, v, ks, vs = op.places(64)
    scales = np.maximum(np.arange(256), 1).astype(np.uint8)
    for row in range(256):
        page, r = c.pool[c.table[0, row // 64]], row % 64
        for at in (k, v):
            page[at[r, 0::2]] = codes[0::2] | codes[1::2] << 4
        page[ks[r]], page[vs[r]] = scales[row], scales[255 - row]
    off = torch.tensor([0, 256], device=DEV)
    back = [torch.empty(256, 64, dtype=c.torch_dtype, device=DEV) for _ in range(2)]
    nkv.pages_read(back[0], back[1], off, 256, c.on(DEV))
    top = torch.finfo(c.torch_dtype).max
    for got, s in zip(back, (scales, scales[::-1])):
        exact = op.values(np.tile(codes, (256, 1)), np.repeat(s[:, None], 2, 1))
        want = torch.from_numpy(np.clip(exact, -top, top)).to(c.torch_dtype)
        differ = (_bits(got) != _bits(want)).nonzero()
        assert differ.numel() == 0, [(int(s[r]), int(codes[d]), float(got[r, d]), float(want[r, d])) for r, d in differ[:6].tolist()]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_the_types_extremes_go_into_4_bits_and_back(dtype):
    """Blocks of the type's largest, smallest normal and subnormal values: the pool's bytes, and the rows' bits after a read."""
    c = Cache(1, 1, 64, dtype, "fp4", [64], seed=31)
    f = torch.finfo(c.torch_dtype)
    x = torch.zeros(64, 64)
    for i, m in enumerate((f.max, f.max / 2, f.tiny, f.tiny / 2, f.smallest_normal * 1.75, f.tiny * 0.75, f.tiny * 0.53125, f.tiny / 4, f.tiny * 7)):
        part = torch.tensor([1.0, 0.875, 0.75, 0.625, 0.5, 0.375, 0.3125, 0.25, 0.1875, 0.125, 0.0625, 0.0])
        x[i, :12], x[i, 16:28], x[i, 32:44] = m * part, -m * part, m * part.flip(0)
    rows = x.to(c.torch_dtype)
    pages, off = c.on(DEV), torch.tensor([0, 64], device=DEV)
    nkv.pages_load(rows.to(DEV), rows.flip(0).contiguous().to(DEV), off, 64, pages)
    torch.cuda.synchronize()
    want, y = c.pool.copy(), _f64(rows)
    for r in range(64):
        op.write_row(want[c.table[0, 0]], r, True, y[r], True, None)
        op.write_row(want[c.table[0, 0]], r, False, y[63 - r], True, None)
    assert np.array_equal(c.d_pool.cpu().numpy(), want)
    k, v = torch.empty_like(rows, device=DEV), torch.empty_like(rows, device=DEV)
    nkv.pages_read(k, v, off, 64, pages)
    for got, exact in zip((k, v), op.read_rows(want[c.table[0, 0]], 64, True, None)):
        assert torch.equal(_bits(got), _bits(torch.from_numpy(np.clip(exact, -f.max, f.max)).to(c.torch_dtype)))


@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt,dtype", [("fp4", "bf16"), ("fp4", "fp16"), ("16bit", "bf16")])
@pytest.mark.parametrize("behind", [0, 37])
def test_load_and_read(d, fmt, dtype, behind):
    """Ragged packed rows to the end of every unit's pages, `behind` rows that are there already, and back: whole pools and rows compared."""
    n = [0, 1, 63, 64, 65, 200, 0, 130]
    c = Cache(4, 2, d, dtype, fmt, [x + behind for x in n], rows=1.0, seed=d + behind)
    off = np.concatenate([[0], np.cumsum(n)])
    rows = int(off[-1])
    g = torch.Generator().manual_seed(d)
    k, v = (torch.randn(rows, d, generator=g).to(c.torch_dtype) for _ in range(2))
    want, bits = c.pool.copy(), to_bits(c.torch_dtype)
    for u in range(8):
        for i in range(n[u]):
            row = behind + i
            for key, x in ((True, k), (False, v)):
                op.write_row(want[c.table[u, row // 64]], row % 64, key, _f64(x[off[u] + i]), c.fp4, bits)
    pages = c.on(DEV)
    d_off = torch.from_numpy(off).to(DEV)
    nkv.pages_load(k.to(DEV), v.to(DEV), d_off, rows, pages)
    torch.cuda.synchronize()
    assert np.array_equal(c.d_pool.cpu().numpy(), want)
    back = [torch.full((rows + 2, d), float("nan"), dtype=c.torch_dtype, device=DEV) for _ in range(2)]
    nkv.pages_read(back[0][1:-1], back[1][1:-1], d_off, rows, pages)
    torch.cuda.synchronize()
    for got, x in zip(back, (k, v)):
        held = op.values(*op.quantise(_f64(x))) if c.fp4 else _f64(x)
        assert np.array_equal(_f64(got[1:-1]), held)
        assert bool(got[0].isnan().all()) and bool(got[-1].isnan().all())


def test_rows_that_have_no_place():
    """More packed rows than a unit has: the front ones are left out, and read as zeros; pages outside the pool are not written and read as zeros; offsets beyond
    the buffer and descending ones are clamped."""
    c = Cache(1, 5, 64, "bf16", "16bit", [70, 40, 130, 10, 5], rows=1.0, seed=11)
    c.table[2, 1] = c.pool.shape[0] + 3
    off = [0, 150, 190, 320, 310, 500]                     # unit 0: 80 rows in front; unit 3: descending; unit 4: clamped to 400
    rows = 400
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(rows, 64, generator=g).to(torch.bfloat16) for _ in range(2))
    want, bits = c.pool.copy(), to_bits(torch.bfloat16)
    held = np.full((2, rows, 64), np.nan)
    for u in range(5):
        a, b = min(off[u], rows), min(off[u + 1], rows)
        for i in range(a, b):
            row = int(c.lens[u]) - (b - a) + i - a
            held[:, i] = 0.0
            if row >= 0 and c.table[u, row // 64] < c.pool.shape[0]:
                for j, x in enumerate((k, v)):
                    op.write_row(want[c.table[u, row // 64]], row % 64, j == 0, _f64(x[i]), False, bits)
                    held[j, i] = _f64(x[i])
    pages = c.on(DEV)
    d_off = torch.tensor(off, device=DEV)
    nkv.pages_load(k.to(DEV), v.to(DEV), d_off, rows, pages)
    torch.cuda.synchronize()
    got = c.d_pool.cpu().numpy()
    page_rows = [(int(c.table[4, 0]), r) for r in range(5)]   # unit 4: 90 rows for 5 places, those of unit 3 among them
    assert np.array_equal(got, want), page_rows
    back = [torch.full((rows, 64), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    nkv.pages_read(back[0], back[1], d_off, rows, pages)
    torch.cuda.synchronize()
    for j in range(2):
        assert np.array_equal(_f64(back[j])[:310], held[j][:310], equal_nan=True)
    nkv.pages_load(k.to(DEV), v.to(DEV), d_off, 0, pages)  # no rows at all
    torch.cuda.synchronize()


def test_many_units_of_few_rows():
    c = Cache(600, 8, 64, "bf16", "16bit", np.arange(4800) % 4, seed=12)
    off = np.concatenate([[0], np.cumsum(c.lens.astype(np.int64))])
    rows = int(off[-1])
    k = torch.randn(rows, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(DEV)
    v, pages, d_off = k * 2, c.on(DEV), torch.from_numpy(off).to(DEV)
    nkv.pages_load(k, v, d_off, rows, pages)
    a, b = torch.empty_like(k), torch.empty_like(k)
    nkv.pages_read(a, b, d_off, rows, pages)
    torch.cuda.synchronize()
    assert torch.equal(a, k) and torch.equal(b, v)


# ---- attention ----

@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (3, 2)])
def test_attention_at_every_edge(d, fmt, dtype, G, n):
    c = Cache(8, 2, d, dtype, fmt, EDGES, rows=1.0, seed=d + G)
    q = _queries(c, n, 2 * G, 3)
    o, l = _attend(c, q, d ** -0.5, n, 2 * G)
    _check(c, q, o, l, d ** -0.5, f"{d} {fmt} {dtype} G={G} n={n}", n)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("G,n", [(2, 1), (5, 1), (8, 1), (16, 1), (20, 1), (33, 1), (4, 4), (8, 5), (1, 17), (16, 3), (6, 7)])
def test_attention_groups_and_tokens(fmt, G, n):
    c = Cache(2, 3, 128, "bf16", fmt, [3, 64, 70, 131, 0, 390], rows=1.0, seed=G)
    q = _queries(c, n, 3 * G, 5)
    o, l = _attend(c, q, 128 ** -0.5, n, 3 * G)
    _check(c, q, o, l, 128 ** -0.5, f"G={G} n={n}", n)


@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (5, 1), (3, 2), (8, 5)])
def test_attention_keeps_every_bit_of_its_weights(d, fmt, dtype, G, n):
    """The bar from the values that are there, at which a lost piece of the weights' split shows (tests/test_pages_host.py)."""
    c = Cache(8, 2, d, dtype, fmt, EDGES, rows=1.0, seed=d + G)
    q = _queries(c, n, 2 * G, 3)
    o, l = _attend(c, q, d ** -0.5, n, 2 * G)
    want, want_lse = op.attention(_f64(q), c.pool, c.table, c.lens, 2, d ** -0.5, d, c.fp4, from_bits(c.torch_dtype))
    err, bar = np.abs(_f64(o) - want).max(), attention_bar(np.abs(values_of(c)).max())
    assert err <= bar, f"out off by {err:.3e}, bar {bar:.3e}"
    seen = np.isfinite(want_lse)
    assert np.array_equal(np.isfinite(_f64(l)), seen) and np.abs(_f64(l)[seen] - want_lse[seen]).max() <= TOL


@pytest.mark.parametrize("fmt,d,dtype", [("fp4", 128, "bf16"), ("16bit", 128, "bf16"), ("fp4", 64, "fp16"), ("16bit", 64, "fp16")])
def test_attention_over_long_and_short_units_together(fmt, d, dtype):
    """One unit of 20 000 rows beside 30 of a few: stretches end inside the long one and run over several of the short ones."""
    c = Cache(31, 1, d, dtype, fmt, [5] * 11 + [20000] + list(range(60, 79)), rows=1.0, seed=13)
    q = _queries(c, 1, 4, 6)
    o, l = _attend(c, q, d ** -0.5, 1, 4)
    _check(c, q, o, l, d ** -0.5, fmt, 1)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_attention_over_many_units(fmt):
    lens = (np.arange(3000) * 7) % 150
    lens[100:400] = 0
    c = Cache(375, 8, 64, "bf16", fmt, lens, rows=1.0, seed=14)
    q = _queries(c, 1, 16, 7)
    o, l = _attend(c, q, 0.125, 1, 16)
    _check(c, q, o, l, 0.125, fmt, 1)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_pages_that_are_none_and_lengths_out_of_range(fmt):
    c = Cache(3, 2, 128, "bf16", fmt, [200, 64, 130, 70, 10, 300], width=5, rows=1.0, seed=15)
    c.table[0, 1], c.table[1, 0], c.table[2, 2], c.table[3, 0] = -1, c.pool.shape[0], 2 ** 31 - 1, -2 ** 31
    c.lens[4], c.lens[5] = -5, 10 ** 9                     # no rows; all that the table's row can hold, some on no page
    c.pool[c.table[5, 4]] = 0                              # its last page's unused rows are rows now
    q = _queries(c, 2, 8, 8)
    o, l = _attend(c, q, 0.1, 2, 8)
    _check(c, q, o, l, 0.1, fmt, 2)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_later_tokens_nan_stays_with_it(fmt, d):
    """Tokens see no row behind their own: a NaN in a later token's key or value reaches only those that see it."""
    n, G = 4, 3
    c = Cache(2, 1, d, "bf16", fmt, [70, 131], rows=1.0, seed=16)
    q = _queries(c, n, G, 9)
    want, _ = op.attention(_f64(q), c.pool, c.table, c.lens, 1, 0.1, d, c.fp4, from_bits(c.torch_dtype))
    x = np.full(d, np.nan)
    op.write_row(c.pool[c.table[0, 1]], 68 - 64, False, x, c.fp4, to_bits(c.torch_dtype))    # value of token 2 of 4
    op.write_row(c.pool[c.table[1, 2]], 129 - 128, True, x, c.fp4, to_bits(c.torch_dtype))   # key
    o, l = _attend(c, q, 0.1, n, G)
    for s in range(2):
        assert np.abs(_f64(o)[s, :2] - want[s, :2]).max() <= TOL * 6
        assert np.isnan(_f64(o)[s, 2:]).all()


@pytest.mark.parametrize("fmt,dtype", [("fp4", "bf16"), ("fp4", "fp16"), ("16bit", "fp16")])
@pytest.mark.parametrize("G,n", [(1, 5), (2, 2), (1, 40)])
def test_a_later_tokens_nan_stays_with_it_in_few_columns_and_over_pages(fmt, dtype, G, n):
    """The same with five columns at most, whose weights' pieces lie side by side, and with more tokens than a half page has rows: NaN in the value of
    one token in the middle, in the key of the next."""
    c = Cache(2, 1, 128, dtype, fmt, [70, 131], rows=1.0, seed=26)
    q = _queries(c, n, G, 9)
    want, want_lse = op.attention(_f64(q), c.pool, c.table, c.lens, 1, 0.1, 128, c.fp4, from_bits(c.torch_dtype))
    t = n // 2
    for s, key in ((0, False), (1, True)):
        row = int(c.lens[s]) - n + t + s
        if row < c.lens[s]:
            op.write_row(c.pool[c.table[s, row // 64]], row % 64, key, np.full(128, np.nan), c.fp4, to_bits(c.torch_dtype))
    o, l = _attend(c, q, 0.1, n, G)
    for s in range(2):
        assert np.abs(_f64(o)[s, :t + s] - want[s, :t + s]).max() <= TOL * 6 and np.abs(_f64(l)[s, :t + s] - want_lse[s, :t + s]).max() <= TOL * 10
        assert np.isnan(_f64(o)[s, t + s:]).all()


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("d,G,n", [(128, 3, 4), (64, 1, 4), (256, 1, 20)])
def test_a_later_tokens_largest_value_stays_with_it(fmt, d, G, n):
    """The value of a token in the middle holds bf16's largest number, which in 4 bits is 2^128: tokens in front of it do not see it."""
    c = Cache(2, 1, d, "bf16", fmt, [70, 131], rows=1.0, seed=28)
    q = _queries(c, n, G, 9)
    want, want_lse = op.attention(_f64(q), c.pool, c.table, c.lens, 1, 0.1, d, c.fp4, from_bits(c.torch_dtype))
    t = n // 2
    for s in range(2):
        row = int(c.lens[s]) - n + t
        x = np.linspace(-1, 1, d)
        x[5], x[d - 1] = torch.finfo(torch.bfloat16).max, -torch.finfo(torch.bfloat16).max
        op.write_row(c.pool[c.table[s, row // 64]], row % 64, False, x, c.fp4, to_bits(c.torch_dtype))
    o, l = _attend(c, q, 0.1, n, G)
    assert np.abs(_f64(o)[:, :t] - want[:, :t]).max() <= TOL * 6 and np.abs(_f64(l)[:, :t] - want_lse[:, :t]).max() <= TOL * 10
    for s in range(2):
        assert (~(np.abs(_f64(o)[s, t:, :, 5]) < 1e30)).all()             # large, infinite or NaN


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_peaked_flat_and_negative_logits(fmt, dtype):
    """One row that takes nearly all weight, all rows alike (scale 0: the mean of the values, lse = log n), a negative scale, large logits."""
    c = Cache(1, 2, 128, dtype, fmt, [500, 130], rows=1.0, seed=17)
    q = _queries(c, 1, 4, 10)
    for scale in (0.0, -0.1, 0.3):
        o, l = _attend(c, q, scale, 1, 4)
        _check(c, q, o, l, scale, str(scale), 1)
    _, l = _attend(c, q, 0.0, 1, 4)
    assert np.allclose(_f64(l)[0, 0], np.log([500, 500, 130, 130]), atol=1e-6)
    big = (q * 30).to(q.dtype)                             # logits of some hundreds: 2^-24 of them, times the roundings of a sum, in the exponent
    o, l = _attend(c, big, 0.088, 1, 4)
    want, want_lse = op.attention(_f64(big), c.pool, c.table, c.lens, 2, 0.088, 128, c.fp4, from_bits(c.torch_dtype))
    assert np.abs(_f64(o) - want).max() <= 6 * 2e-3 and np.abs(_f64(l) / want_lse - 1).max() <= TOL


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_queries_of_very_different_sizes(fmt):
    """Small query values beside large ones keep their share: dims whose keys are zero hold the large ones."""
    c = Cache(1, 1, 128, "bf16", fmt, [64], rows=1.0, seed=18)
    page = c.pool[c.table[0, 0]]
    K, V = op.read_rows(page, 128, c.fp4, from_bits(c.torch_dtype))
    for r in range(64):
        K[r, :32] = 0.0
        op.write_row(page, r, True, K[r], c.fp4, to_bits(c.torch_dtype))
    q = _queries(c, 1, 1, 11)
    q[..., :32] *= 500
    o, l = _attend(c, q, 0.2, 1, 1)
    _check(c, q, o, l, 0.2, fmt, 1)


def _times_power_of_two(c, key, e):
    """The K (or V) rows of all units times 2^e."""
    k, v, ks, vs = op.places(c.d)
    for u, n in enumerate(c.lens):
        for j in range((int(n) + 63) // 64):
            page, m = c.pool[c.table[u, j]], min(64, int(n) - 64 * j)
            if c.fp4:
                page[(ks if key else vs)[:m]] += np.uint8(e)
            else:
                w = page.view(np.uint16).reshape(2, 64, c.d)[0 if key else 1]
                w[:m] = to_bits(c.torch_dtype)(from_bits(c.torch_dtype)(w[:m].reshape(-1)) * 2.0 ** e).reshape(m, c.d)


@pytest.mark.parametrize("fmt,dtype", [("fp4", "bf16"), ("fp4", "fp16"), ("16bit", "bf16")])
@pytest.mark.parametrize("up,scale", [(56, 0.0), (56, 0.09 * 2.0 ** -113), (56, -0.09 * 2.0 ** -113), (59, 0.09 * 2.0 ** -119), (59, 0.09 * 2.0 ** -128), (59, 2.0 ** -160)])
def test_scales_far_below_one_beside_large_products(fmt, dtype, up, scale):
    """Logits of ordinary size from products of up to 2^125, also by a scale that is subnormal in fp32, and a scale (zero, or as good as) by which all rows weigh the same."""
    c = Cache(2, 2, 128, dtype, fmt, [200, 33, 64, 1], rows=1.0, seed=24)
    up_q = up if dtype == "bf16" else 8
    _times_power_of_two(c, True, up + 1 + (up - up_q))
    q = (_queries(c, 1, 8, 15).double() * 2.0 ** up_q).to(c.torch_dtype)
    o, l = _attend(c, q, scale, 1, 8)
    _check(c, q, o, l, scale, str((up, scale)), 1)


@pytest.mark.parametrize("fmt,dtype,e_k,e_q", [("fp4", "bf16", 20, 18), ("fp4", "fp16", 30, 10), ("16bit", "bf16", 20, 18), ("16bit", "fp16", 11, 11)])
@pytest.mark.parametrize("d,G", [(128, 4), (64, 8), (256, 3)])
def test_logits_of_millions_give_the_largest_ones_row(fmt, dtype, e_k, e_q, d, G):
    """Logits between which lie more than 2^20: the weight of all rows but one is 0 in any precision, and where a step of the logits in fp32 is more than a few units, so that
    the running maximum is off by as much, weights stay finite all the same.  Rows are a_i times one vector of signs, with a_i = 6 in one row and up to 4 in the others."""
    c = Cache(2, 2, d, dtype, fmt, [70, 300, 33, 129], rows=1.0, seed=25 + d)
    g = torch.Generator().manual_seed(d)
    signs = torch.where(torch.randn(d, generator=g) < 0, -1.0, 1.0).double().numpy()
    best = []
    for u, n in enumerate(c.lens):
        a = np.array([1.0, 1.5, 2.0, 3.0, 4.0])[torch.randint(0, 5, (int(n),), generator=g).numpy()]
        best.append(int(torch.randint(0, int(n), (1,), generator=g)))
        a[best[u]] = 6.0
        for i in range(int(n)):
            op.write_row(c.pool[c.table[u, i // 64]], i % 64, True, a[i] * 2.0 ** e_k / 4 * signs, c.fp4, to_bits(c.torch_dtype))
    # every query a size of its own, so that the logits' roundings differ
    size = 1.0 + torch.randint(0, 64, (2, 1, 2 * G, 1), generator=g).double() / 64
    q = (size * 2.0 ** e_q / 2 * torch.from_numpy(signs)).to(c.torch_dtype)
    for scale in (d ** -0.5, 1.0):
        o, l = _attend(c, q, scale, 1, 2 * G)
        want, want_lse = op.attention(_f64(q), c.pool, c.table, c.lens, 2, scale, d, c.fp4, from_bits(c.torch_dtype))
        assert want_lse.min() > 2.0 ** 20
        assert np.isfinite(_f64(o)).all() and np.isfinite(_f64(l)).all()
        # one row's values: the split of its weight is all that is rounded, and the sum that it is divided by
        assert (np.abs(_f64(o) - want) <= 2.0 ** -20 * np.abs(want)).all()
        assert np.abs(_f64(l) / want_lse - 1).max() <= TOL


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
@pytest.mark.parametrize("n", [5, 16])
def test_tokens_without_rows_leave_the_others_weights_as_they_are(fmt, n):
    """Logits of some hundreds, a few apart: in a call whose first tokens see no row, a token's weights are those of a call of its own (whose products are the
    same sums in fp32), to a few roundings; logits rounded before the maximum is taken from them would be 1.5e-5 off."""
    d, rows = 64, 4
    c = Cache(1, 1, d, "bf16", fmt, [rows], rows=1.0, seed=27)
    g = torch.Generator().manual_seed(4)
    mean = torch.randn(d, generator=g).sign().double().numpy() * 3.0
    K = mean + 0.25 * torch.randn(rows, d, generator=g).double().numpy()
    for i in range(rows):
        op.write_row(c.pool[c.table[0, 0]], i, True, K[i], c.fp4, to_bits(c.torch_dtype))
    q = torch.from_numpy(mean * (1 + 0.1 * torch.rand(1, n, 1, d, generator=g).double().numpy())).to(c.torch_dtype)
    scale = 0.5
    o, l = _attend(c, q, scale, n, 1)
    for t in range(n - rows, n):
        alone = Cache(1, 1, d, "bf16", fmt, [rows], seed=27)
        alone.pool, alone.table, alone.lens = c.pool, c.table, np.array([rows - (n - 1 - t)], np.int32)
        o1, l1 = _attend(alone, q[:, t:t + 1].contiguous(), scale, 1, 1)
        assert float(l1) > 200
        assert np.abs(_f64(o)[0, t] - _f64(o1)[0, 0]).max() <= 2e-6, t
    assert bool((o[0, :n - rows] == 0).all()) and bool(l[0, :n - rows].isneginf().all())


def test_units_may_share_pages():
    c = Cache(4, 1, 64, "bf16", "fp4", [130, 100, 64, 130], rows=1.0, seed=19)
    c.table[1:] = c.table[0]
    q = _queries(c, 1, 2, 12)
    o, l = _attend(c, q, 0.125, 1, 2)
    _check(c, q, o, l, 0.125, "shared", 1)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_calls_repeat_bit_for_bit_on_any_stream_and_without_lse(fmt):
    c = Cache(5, 2, 128, "bf16", fmt, [900, 64, 1, 0, 300, 2000, 77, 128, 129, 5], rows=1.0, seed=20)
    q = _queries(c, 2, 8, 13)
    o, l = _attend(c, q, 0.09, 2, 8)
    other = torch.cuda.Stream()
    o2, l2 = _attend(c, q, 0.09, 2, 8, stream=other)
    o3, _ = _attend(c, q, 0.09, 2, 8, want_lse=False)
    assert torch.equal(o, o2) and torch.equal(o, o3) and torch.equal(l, l2)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB: pages at its far end."""
    d, far = 256, (1 << 32) // op.page_bytes(256, False) + 100
    c = Cache(1, 1, d, "bf16", "16bit", [150], rows=1.0, seed=21)
    pool = torch.full((far + 3, op.page_bytes(d, False)), 255, dtype=torch.uint8, device=DEV)
    pool[far:far + 3] = torch.from_numpy(c.pool[c.table[0]]).to(DEV)
    table = torch.arange(far, far + 3, dtype=torch.int32, device=DEV)[None]
    lens = torch.tensor([150], dtype=torch.int32, device=DEV)
    pages = nkv.Pages(1, 1, d, nkv.DTYPE_BF16, nkv.PAGES_16BIT, pool, table, lens)
    q = _queries(c, 1, 2, 14)
    out, ws = torch.empty(1, 1, 2, d, device=DEV), torch.empty(nkv.pages_workspace_bytes(pages, 2), dtype=torch.uint8, device=DEV)
    nkv.pages_attention(q.to(DEV), pages, 2, 1, 0.06, out, None, ws)
    _check(c, q, out, None, 0.06, "far", 1)
    k, v = torch.empty(150, d, dtype=torch.bfloat16, device=DEV), torch.empty(150, d, dtype=torch.bfloat16, device=DEV)
    off = torch.tensor([0, 150], device=DEV)
    nkv.pages_read(k, v, off, 150, pages)
    nkv.pages_load(v, k, off, 150, pages)                   # swapped
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    nkv.pages_read(k2, v2, off, 150, pages)
    assert torch.equal(k, v2) and torch.equal(v, k2)


# ---- together ----

@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_captured_decode_steps_replay(fmt):
    """Three decode steps (lens + 1, append, attention) recorded once: every replay goes on from where the last one stopped, and eager steps from the
    same start give the same bits."""
    S, H, G, d, steps = 3, 2, 4, 128, 4
    c = Cache(S, H, d, "bf16", fmt, [60, 61, 62, 63, 64, 10], width=4, rows=1.0, seed=22)
    spare = np.full((S * H, c.pool.shape[1]), 255, np.uint8)   # a page more for every unit
    for u in range(S * H):
        c.table[u, (int(c.lens[u]) + 63) // 64] = c.pool.shape[0] + u
    c.pool = np.concatenate([c.pool, spare])
    rope = nkv.rope_table(200, d, device=DEV)
    x = torch.randn(S, 1, (G + 2) * H, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)

    def state():
        pages = c.on(DEV)
        s = dict(pages=pages, lens=c.d_lens, pool=c.d_pool, pos=torch.tensor([[100], [90], [80]], dtype=torch.int32, device=DEV))
        s["q"] = torch.empty(S, 1, G * H, d, dtype=torch.bfloat16, device=DEV)
        s["out"], s["lse"] = torch.empty(S, 1, G * H, d, device=DEV), torch.empty(S, 1, G * H, device=DEV)
        s["ws"] = torch.empty(nkv.pages_workspace_bytes(pages, G * H), dtype=torch.uint8, device=DEV)
        return s

    def step(s):
        s["lens"] += 1
        nkv.pages_append(x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:], s["pages"], positions=s["pos"], rope=rope, q=x[:, :, :G * H], q_out=s["q"])
        nkv.pages_attention(s["q"], s["pages"], G * H, 1, d ** -0.5, s["out"], s["lse"], s["ws"])
        s["pos"] += 1

    eager, caught = state(), state()
    wanted = []
    for _ in range(steps):
        step(eager)
        wanted.append((eager["out"].clone(), eager["lse"].clone()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(caught)
    for out, lse in wanted:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(caught["out"], out) and torch.equal(caught["lse"], lse)
        float(x.float().sum())                              # the program's own work in between
    assert torch.equal(caught["pool"], eager["pool"]) and torch.equal(caught["lens"], eager["lens"])
    c.pool, c.lens = eager["pool"].cpu().numpy(), eager["lens"].cpu().numpy()
    _check(c, eager["q"], eager["out"], eager["lse"], d ** -0.5, "after the last step", 1)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_the_compressors_rows_through_pages(fmt):
    """compress -> load -> attend; 16-bit pages agree with attention over the packed rows themselves."""
    w = nkv_inputs.small_workload("pages", 2, 2, 128, [700, 333])
    K, V = nkv_inputs.make_kv(w, "cpu")
    shape = shape_of(w)
    comp = nkv.Compressor(shape, [0.6, 0.5])
    r = comp.run(K.to(DEV), V.to(DEV))
    lens = (r.head_off[1:] - r.head_off[:-1]).int()
    c = Cache(4, 2, 128, "bf16", fmt, lens.cpu().numpy(), seed=23)
    pages = c.on(DEV)
    nkv.pages_load(r.packed_k, r.packed_v, r.head_off, comp.rows, pages)
    q = nkv_inputs.make_queries(w, 8, K).to(DEV)             # [P, L, Hq, d]: sequence p * L + l
    out = torch.empty(4, 1, 8, 128, device=DEV)
    lse = torch.empty(4, 1, 8, device=DEV)
    ws = torch.empty(nkv.pages_workspace_bytes(pages, 8), dtype=torch.uint8, device=DEV)
    nkv.pages_attention(q.reshape(4, 1, 8, 128), pages, 8, 1, 128 ** -0.5, out, lse, ws)
    torch.cuda.synchronize()
    c.pool = c.d_pool.cpu().numpy()
    _check(c, q.reshape(4, 1, 8, 128), out, lse, 128 ** -0.5, fmt, 1)
    if fmt == "16bit":
        want, want_lse = torch.empty(2, 2, 8, 128, device=DEV), torch.empty(2, 2, 8, device=DEV)
        ws2 = torch.empty(max(256, nkv.decode_workspace_bytes(shape, 8, comp.rows)), dtype=torch.uint8, device=DEV)
        nkv.decode_attention(q, r.packed_k, r.packed_v, r.head_off, comp.rows, shape, comp.params, 8, 128 ** -0.5, want, want_lse, ws2)
        torch.cuda.synchronize()
        assert float((out.reshape(want.shape) - want).abs().max()) <= 2 * TOL * 6
        assert float((lse.reshape(want_lse.shape) - want_lse).abs().max()) <= 2 * TOL * 10


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_a_cache_that_grows_and_gives_back_while_it_decodes_layer_by_layer(fmt):
    """Steps of all layers in one graph.  Pages are reserved as units fill theirs; in the middle a prompt is released, its pages go to the others, and another
    prompt comes into its place.  After every step each layer's output is that of the rows appended so far, by the oracle."""
    P, L, H, G, d, steps = 3, 2, 2, 2, 64, 12
    Hq, scale = G * H, d ** -0.5
    c = nkv.PagedCache(P * L, H, d, nkv.DTYPE_BF16, nkv.PAGES_FP4 if fmt == "fp4" else nkv.PAGES_16BIT, n_pages=27, max_rows=200, device=DEV)
    lens = [60, 61, 125, 58, 3, 64, 62, 63, 1, 120, 59, 57]
    assert len(lens) == P * L * H
    g = torch.Generator().manual_seed(5)

    def fill(units, n):                                     # packed rows into those units' pages
        off = np.concatenate([[0], np.cumsum([n[u] if u in units else 0 for u in range(P * L * H)])])
        k, v = (torch.randn(int(off[-1]), d, generator=g).to(torch.bfloat16) for _ in range(2))
        c.lens.copy_(torch.tensor(n, dtype=torch.int32))
        nkv.pages_load(k.to(DEV), v.to(DEV), torch.from_numpy(off).to(DEV), int(off[-1]), c.pages)

    c.reserve(lens)
    fill(range(P * L * H), lens)
    layers = c.layers(L)
    qkv = torch.empty(L, P, 1, Hq + 2 * H, d, dtype=torch.bfloat16, device=DEV)
    q = torch.empty(L, P, 1, Hq, d, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.empty(L, P, 1, Hq, d, device=DEV), torch.empty(L, P, 1, Hq, device=DEV)
    rope, positions = nkv.rope_table(400, d, device=DEV), torch.tensor([[70], [80], [90]], dtype=torch.int32, device=DEV)
    alive = torch.ones(P * H, dtype=torch.int32, device=DEV)
    ws = torch.empty(nkv.pages_workspace_bytes(layers[0], Hq), dtype=torch.uint8, device=DEV)

    def step():
        c.layer_lens.add_(alive)
        positions.add_(1)
        for l in range(L):
            x = qkv[l]
            nkv.pages_append(x[:, :, Hq:Hq + H], x[:, :, Hq + H:], layers[l], positions=positions, rope=rope, q=x[:, :, :Hq], q_out=q[l])
            nkv.pages_attention(q[l], layers[l], Hq, 1, scale, out[l], lse[l], ws)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    lens, live = np.array(lens), np.ones(P * L * H, int)
    bits, halves = to_bits(torch.bfloat16), True
    for t in range(steps):
        if t == 5:                                          # prompt 1 ends
            for l in range(L):
                c.release(1 * L + l)
            alive.view(P, H)[1] = 0
            positions[1] = -1000
            live.reshape(P, L, H)[1], lens.reshape(P, L, H)[1] = 0, 0
        if t == 8:                                          # another one in its place
            n = lens.copy()
            n.reshape(P, L, H)[1] = [[30, 70], [64, 1]]
            c.reserve(n.tolist())
            fill([u for u in range(P * L * H) if u // H // L == 1], n.tolist())
            c.layer_lens.view(L, P, H)[:, 1] = torch.from_numpy(n.reshape(P, L, H)[1]).int().to(DEV)
            alive.view(P, H)[1] = 1
            positions[1] = 100
            lens, live = n, np.ones(P * L * H, int)
        lens = lens + live
        c.reserve(lens.tolist())
        x = torch.randn(L, P, 1, Hq + 2 * H, d, generator=g).to(torch.bfloat16)
        qkv.copy_(x)
        pos = positions.cpu().numpy() + 1
        before = c.pool.cpu().numpy()
        table = c.table.cpu().numpy()
        held = table[table >= 0]
        assert len(set(held.tolist())) == held.size         # every page is one unit's
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.layer_lens.cpu().view(L, P, H), torch.from_numpy(lens).int().view(P, L, H).transpose(0, 1)), t
        for l in range(L):
            f = _f64(x[l])
            turned = op.rotate(f[:, :, :Hq + H], pos, rope.cpu().numpy(), halves)
            for u in np.flatnonzero(live.reshape(P, L, H)[:, l].reshape(-1)):
                p, h = divmod(int(u), H)
                unit = (p * L + l) * H + h
                row = int(lens[unit]) - 1
                page = before[table[unit, row // 64]]
                op.write_row(page, row % 64, True, turned[p, 0, Hq + h], fmt == "fp4", bits)
                op.write_row(page, row % 64, False, f[p, 0, Hq + H + h], fmt == "fp4", bits)
            of = table.reshape(P, L, H, -1)[:, l].reshape(P * H, -1)
            n = lens.reshape(P, L, H)[:, l].reshape(-1)
            seen = from_bits(torch.bfloat16)(bits(turned[:, :, :Hq]).reshape(-1)).reshape(P, 1, Hq, d)
            want, want_lse = op.attention(seen, before, of, n, H, scale, d, fmt == "fp4", from_bits(torch.bfloat16))
            assert np.abs(_f64(out[l]) - want).max() <= TOL * 6, (t, l)
            assert np.array_equal(np.isneginf(_f64(lse[l])), np.isneginf(want_lse)), (t, l)
        assert np.array_equal(c.pool.cpu().numpy(), before), t


_FORM = dict(dtype="bf16", fmt="fp4", H=8, G=4, d=128)


@pytest.mark.parametrize("case", [
    dict(_FORM, path="append", S=2, n=40, held=100, rot=128, style="halves"),
    dict(_FORM, path="append", S=2, n=33, held=0, rot=48, style="pairs", H=32, G=1, d=96, dtype="fp16", fmt="16bit"),
    dict(_FORM, path="load", S=3, rows=150, uneven=True),
    dict(_FORM, path="load", S=3, rows=70, uneven=True, d=256, dtype="fp16"),
    dict(_FORM, path="attend", S=2, rows=300, uneven=True, n=1),
    dict(_FORM, path="attend", S=2, rows=200, uneven=True, n=4, G=3, d=64, fmt="16bit"),
    dict(_FORM, path="attend", S=2, rows=200, uneven=True, n=2, G=8, dtype="fp16"),
    dict(_FORM, path="step", S=3, rows=260, uneven=True, n=1, rot=128, style="halves"),
], ids=lambda c: "-".join(str(x) for x in c.values()))
def test_plain_form_definition_and_calls_agree(case, monkeypatch):
    """The forms that perf/operators.py times, on small cases: rows bit for bit, attention against 64 bits."""
    from perf import operators
    monkeypatch.setattr(operators, "own", False)
    plain = operators.run(operators.prepare(case, 3))
    plain = {x: t.clone() for x, t in plain.items()}
    exact = operators.exact(case, 3)
    monkeypatch.setattr(operators, "own", True)
    own = operators.run(operators.prepare(case, 3))
    torch.cuda.synchronize()
    assert set(own) == set(plain) == set(exact)
    for x, t in own.items():
        assert t.shape == plain[x].shape and t.dtype == plain[x].dtype
        if x in "qkv":
            assert torch.equal(t, plain[x]), x
        else:
            bar = attention_bar(6.0) if x == "attn" else TOL * 16           # V: normal rows; sums of weights up to e^16
            for y in (t, plain[x]):
                y, want = y.double(), exact[x]
                assert torch.equal(y.isneginf(), want.isneginf()) and float((y - want).nan_to_num(0.0).abs().max()) <= bar, x


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_the_example_runs(fmt, monkeypatch, capsys):
    import importlib.util
    import os
    import sys
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")
    spec = importlib.util.spec_from_file_location("paged_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", [path, "--format", fmt, "--prompt", "700", "--tokens", "6", "--layers", "2"])
    assert example.main() == 0
    assert f"{fmt} pages hold" in capsys.readouterr().out
