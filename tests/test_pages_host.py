"""The paged cache without a GPU: what its calls refuse, its sizes, and the oracle's layout and 4-bit format."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import pages as op
import paper_2605_26678_amd as nkv

FAKE = 4096                              # never dereferenced: every call below must fail in validation


def _pages(**kw):
    p = dict(struct_size=C.sizeof(nkv.nkv_pages), n_seqs=2, H=4, d=128, dtype=nkv.DTYPE_BF16, format=nkv.PAGES_FP4, n_pages=10, max_pages=5,
             pool=FAKE, table=FAKE, lens=FAKE)
    p.update(kw)
    return nkv.nkv_pages(*[p[f] for f, _ in nkv.nkv_pages._fields_])


def _tokens(**kw):
    s = lambda *x: (C.c_int64 * 3)(*x)  # noqa: E731
    t = dict(struct_size=C.sizeof(nkv.nkv_tokens), n_new=3, n_q_heads=8, rot=128, rope_style=nkv.ROPE_HALVES, n_positions=100, k=FAKE, v=FAKE, q=FAKE,
             q_out=2 * FAKE, k_strides=s(2048, 512, 128), v_strides=s(2048, 512, 128), q_strides=s(4096, 1024, 128), positions=FAKE, rope=FAKE)
    t.update(kw)
    return nkv.nkv_tokens(*[t[f] for f, _ in nkv.nkv_tokens._fields_])


BAD_PAGES = [
    (dict(struct_size=4), nkv.NKV_EINVAL), (dict(dtype=7), nkv.NKV_EINVAL), (dict(format=2), nkv.NKV_EINVAL), (dict(format=-1), nkv.NKV_EINVAL),
    (dict(pool=0), nkv.NKV_EINVAL), (dict(pool=FAKE + 8), nkv.NKV_EINVAL), (dict(table=0), nkv.NKV_EINVAL), (dict(lens=0), nkv.NKV_EINVAL),
    (dict(lens=FAKE + 2), nkv.NKV_EINVAL), (dict(n_seqs=0), nkv.NKV_ESHAPE), (dict(H=0), nkv.NKV_ESHAPE), (dict(H=33), nkv.NKV_ESHAPE),
    (dict(n_pages=0), nkv.NKV_ESHAPE), (dict(max_pages=0), nkv.NKV_ESHAPE), (dict(d=0), nkv.NKV_ESHAPE), (dict(n_seqs=1 << 20, H=32, max_pages=64), nkv.NKV_ESHAPE),
    (dict(d=80), nkv.NKV_EUNSUPPORTED), (dict(d=32), nkv.NKV_EUNSUPPORTED), (dict(d=512), nkv.NKV_EUNSUPPORTED),
    (dict(dtype=nkv.DTYPE_F32), nkv.NKV_EUNSUPPORTED), (dict(dtype=nkv.DTYPE_F8_E4M3), nkv.NKV_EUNSUPPORTED),
]


@pytest.mark.parametrize("bad", BAD_PAGES, ids=lambda b: str(b)[:40])
def test_every_call_refuses_bad_pages(bad):
    L, (kw, status) = nkv.lib(), bad
    p, t, n = _pages(**kw), _tokens(), C.c_size_t(0)
    assert L.nkv_pages_append(C.byref(t), C.byref(p), 0) == status
    assert L.nkv_pages_load(FAKE, FAKE, FAKE, 10, C.byref(p), 0) == status
    assert L.nkv_pages_read(FAKE, FAKE, FAKE, 10, C.byref(p), 0) == status
    assert L.nkv_pages_workspace_bytes(C.byref(p), 8, 1, C.byref(n)) == status
    assert L.nkv_pages_attention(FAKE, C.byref(p), 8, 1, 1.0, FAKE, 0, FAKE, 1 << 40, 0) == status


@pytest.mark.parametrize("kw", [
    dict(struct_size=0), dict(n_new=0), dict(n_q_heads=-4), dict(n_q_heads=6), dict(k=0), dict(v=0), dict(q=0), dict(q_out=0), dict(q_out=FAKE),
    dict(k=FAKE + 8), dict(q_out=2 * FAKE + 2), dict(rot=24), dict(rot=-16), dict(rot=144), dict(positions=0), dict(rope=0), dict(n_positions=0),
    dict(rope_style=2), dict(positions=FAKE + 2), dict(rope=FAKE + 8), dict(k_strides=(C.c_int64 * 3)(2048, 512, 100)),
    dict(q_strides=(C.c_int64 * 3)(2048, 513, 128)),
], ids=str)
def test_append_refuses_bad_tokens(kw):
    assert nkv.lib().nkv_pages_append(C.byref(_tokens(**kw)), C.byref(_pages()), 0) == nkv.NKV_EINVAL


def test_the_other_calls_refuse_bad_arguments():
    L, p, n = nkv.lib(), _pages(), C.c_size_t(0)
    assert L.nkv_pages_append(None, C.byref(p), 0) == nkv.NKV_EINVAL
    assert L.nkv_pages_append(C.byref(_tokens(n_new=1 << 30)), C.byref(p), 0) == nkv.NKV_ESHAPE
    for call in (L.nkv_pages_load, L.nkv_pages_read):
        assert call(0, FAKE, FAKE, 1, C.byref(p), 0) == nkv.NKV_EINVAL
        assert call(FAKE, FAKE + 2, FAKE, 1, C.byref(p), 0) == nkv.NKV_EINVAL
        assert call(FAKE, FAKE, 0, 1, C.byref(p), 0) == nkv.NKV_EINVAL
        assert call(FAKE, FAKE, FAKE, -1, C.byref(p), 0) == nkv.NKV_EINVAL
        assert call(FAKE, FAKE, FAKE, 1 << 40, C.byref(p), 0) == nkv.NKV_ESHAPE
        assert call(FAKE, FAKE, FAKE, 1, None, 0) == nkv.NKV_EINVAL
    assert L.nkv_pages_workspace_bytes(C.byref(p), 8, 1, None) == nkv.NKV_EINVAL
    for heads, new, status in ((2, 1, nkv.NKV_EINVAL), (6, 1, nkv.NKV_EINVAL), (8, 0, nkv.NKV_EINVAL), (8, 1 << 20, nkv.NKV_ESHAPE)):
        assert L.nkv_pages_workspace_bytes(C.byref(p), heads, new, C.byref(n)) == status
        assert L.nkv_pages_attention(FAKE, C.byref(p), heads, new, 1.0, FAKE, 0, FAKE, 1 << 40, 0) == status
    assert L.nkv_pages_workspace_bytes(C.byref(p), 8, 1, C.byref(n)) == 0 and n.value > 0
    for args in ((0, 1.0, FAKE, 0), (FAKE, float("nan"), FAKE, 0), (FAKE, 1.0, 0, 0), (FAKE + 2, 1.0, FAKE, 0), (FAKE, 1.0, FAKE, 2)):
        q, scale, out, lse = args
        assert L.nkv_pages_attention(q, C.byref(p), 8, 1, scale, out, lse, FAKE, n.value, 0) == nkv.NKV_EINVAL
    for ws, size in ((0, n.value), (FAKE + 16, n.value), (FAKE, n.value - 1)):
        assert L.nkv_pages_attention(FAKE, C.byref(p), 8, 1, 1.0, FAKE, 0, ws, size, 0) == nkv.NKV_EWORKSPACE


def test_calls_that_one_launch_cannot_hold_are_refused():
    # a launch has less than 2^32 threads along x: 256 a token of an append and an output row of the attention, 2 d a page of packed rows
    L, n, top = nkv.lib(), C.c_size_t(0), 1 << 24
    for n_seqs, n_new in ((1, top), (2, top // 2), (top // 8, 8)):
        assert L.nkv_pages_append(C.byref(_tokens(n_new=n_new)), C.byref(_pages(n_seqs=n_seqs, H=1, max_pages=1)), 0) == nkv.NKV_ESHAPE
    for d in (64, 96, 128, 192, 256):
        pages = -(-(1 << 32) // (2 * d))
        p = _pages(n_seqs=1, H=1, d=d)
        for call in (L.nkv_pages_load, L.nkv_pages_read):
            assert call(FAKE, FAKE, FAKE, (pages - 2) * nkv.PAGE_ROWS, C.byref(p), 0) == nkv.NKV_ESHAPE
    for n_seqs, heads, new, status in ((1 << 15, 32, 16, nkv.NKV_ESHAPE), (1 << 15, 32, 15, 0), (1 << 18, 64, 1, nkv.NKV_ESHAPE), ((1 << 18) - 1, 64, 1, 0)):
        p = _pages(n_seqs=n_seqs, H=32, max_pages=1)
        assert L.nkv_pages_workspace_bytes(C.byref(p), heads, new, C.byref(n)) == status
        if status:
            assert L.nkv_pages_attention(FAKE, C.byref(p), heads, new, 1.0, FAKE, 0, FAKE, 1 << 50, 0) == status


def test_binding_refuses_what_the_library_cannot_see():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    table, lens = z(2, 3, dt=torch.int32), z(2, dt=torch.int32)
    pool = z(4, nkv.page_bytes(64, nkv.DTYPE_BF16, nkv.PAGES_FP4), dt=torch.uint8)
    make = lambda **k: nkv.Pages(**{**dict(n_seqs=1, H=2, d=64, dtype=nkv.DTYPE_BF16, format=nkv.PAGES_FP4, pool=pool, table=table, lens=lens), **k})  # noqa: E731
    pages = make()
    assert pages.c.n_pages == 4 and pages.c.max_pages == 3
    for bad in (dict(table=table.long()), dict(lens=lens.long()), dict(table=table[:1]), dict(pool=pool[0, :100]), dict(table=table.T.contiguous().T), dict(H=3)):
        with pytest.raises(ValueError):
            make(**bad)
    with pytest.raises(nkv.NkvError):
        make(d=80)
    k, q, pos, rope = z(1, 3, 2, 64), z(1, 3, 4, 64), z(1, 3, dt=torch.int32), z(9, 2, 32, dt=torch.float32)
    good = dict(k=k, v=k, positions=pos, rope=rope, q=q, q_out=torch.zeros_like(q), stream=0)
    for bad in (dict(k=k.half()), dict(v=z(1, 2, 2, 64)), dict(q=z(1, 3, 4, 128)), dict(q_out=None), dict(q_out=z(1, 3, 4, 128)[..., ::2]),
                dict(rope=rope.double()), dict(positions=pos.long()), dict(rope=rope[:, 0]), dict(positions=pos[:, :2]), dict(k=z(1, 3, 2, 128)[..., ::2])):
        with pytest.raises(ValueError):
            nkv.pages_append(pages=pages, **{**good, **bad})
    with pytest.raises(ValueError):
        nkv.pages_attention(q.half(), pages, 4, 3, 1.0, q, stream=0)
    with pytest.raises(ValueError):
        nkv.pages_load(k.half(), k, lens, 1, pages, stream=0)


def test_sizes():
    for d in (64, 96, 128, 192, 256):
        for dtype in (nkv.DTYPE_BF16, nkv.DTYPE_F16):
            assert nkv.page_bytes(d, dtype, nkv.PAGES_FP4) == op.page_bytes(d, True) and op.page_bytes(d, True) % 16 == 0
            assert nkv.page_bytes(d, dtype, nkv.PAGES_16BIT) == op.page_bytes(d, False)
    for bad in ((80, 1, 1), (128, 0, 1), (128, 3, 0), (128, 1, 2), (-64, 1, 1)):
        assert nkv.page_bytes(*bad) == -1


@pytest.mark.parametrize("d", [64, 96, 128, 192, 256])
def test_every_byte_of_a_4_bit_page_has_one_place(d):
    k, v, ks, vs = op.places(d)
    count = np.zeros(op.page_bytes(d, True), int)
    for codes in (k, v):
        assert np.array_equal(codes[:, 0::2], codes[:, 1::2])              # two neighbouring dims a byte
        np.add.at(count, codes[:, 0::2], 1)
    for scales in (ks, vs):
        np.add.at(count, scales, 1)
    assert (count == 1).all()


def test_4_bit_format_by_hand():
    x = np.zeros((1, 64))
    x[0, :8] = [6.9, 0.25, 0.26, 0.75, 1.25, 2.5, -3.5, -5.0]
    x[0, 32:34] = [7.0, 3.0]
    codes, scales = op.quantise(x)
    assert list(scales[0]) == [127, 128]                                   # 6.9 < 7; 7 takes the next power
    assert list(codes[0, :8]) == [7, 0, 1, 2, 2, 4, 14, 14]
    assert list(codes[0, 32:34]) == [6, 3]                                 # 3.5 and 1.5
    assert list(op.values(codes, scales)[0, :8]) == [6.0, 0.0, 0.5, 1.0, 1.0, 2.0, -4.0, -4.0]
    codes, scales = op.quantise(np.array([[0.0] * 32, [2.0 ** -133] * 32, [np.inf] + [1.0] * 31]))
    assert list(scales[:, 0]) == [1, 1, 255] and not codes.any()
    assert np.isnan(op.values(codes, scales)[2]).all()


def test_quantised_values_are_within_half_a_step():
    """Half of a code's distance to its neighbour (2^s for the largest magnitudes, from 4 * 2^s on), half of 2^s / 2 for the smallest; and
    the scale is the least one that leaves the largest magnitude under 7."""
    x = np.random.RandomState(1).standard_t(3, (50, 96))
    codes, scales = op.quantise(x)
    f = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    step = np.where(np.abs(x) < 2 * f, 0.5, np.where(np.abs(x) < 4 * f, 1.0, 2.0)) * f
    assert (np.abs(op.values(codes, scales) - x) <= step / 2 + 1e-15).all()
    top = np.abs(x).reshape(50, 3, 32).max(-1)
    s = 2.0 ** (scales.astype(float) - 127)
    assert (top < 7 * s).all() and (top >= 3.5 * s).all()


def test_rotation_keeps_lengths_and_differences():
    r = np.random.RandomState(2)
    x = r.randn(1, 2, 1, 64)
    rope = nkv.rope_table(5000, 64, device="cpu").numpy()
    for halves in (True, False):
        y = op.rotate(x, np.array([[3, 4003]]), rope, halves)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-6)
        z = op.rotate(x, np.array([[7, 4007]]), rope, halves)                # the product depends on the difference alone
        assert np.isclose((y[0, 0] * y[0, 1]).sum(), (z[0, 0] * z[0, 1]).sum(), atol=1e-5)
    assert np.allclose(rope[1, 0], np.cos(10000.0 ** (-np.arange(0, 64, 2) / 64)), atol=1e-7)


def test_oracle_attention_is_softmax_attention():
    from pages_util import Cache, from_bits
    c = Cache(2, 2, 64, "bf16", "16bit", [70, 3, 0, 64], rows=1.0, seed=3)
    q = np.random.RandomState(4).randn(2, 2, 4, 64)
    out, lse = op.attention(q, c.pool, c.table, c.lens, 2, 0.125, 64, False, from_bits(c.torch_dtype))
    pages = from_bits(c.torch_dtype)(c.pool.view(np.uint16)).reshape(-1, 2, 64, 64)
    kv = np.concatenate([pages[c.table[0, 0]], pages[c.table[0, 1]]], 1)
    for t in range(2):
        n = 70 - (1 - t)
        k, v = (torch.from_numpy(kv[i][:n]) for i in (0, 1))
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[0, t, :2]), k, v, scale=0.125)
        assert np.allclose(out[0, t, :2], want.numpy(), atol=1e-12)
    assert np.isneginf(lse[1, :, :2]).all() and (out[1, :, :2] == 0).all() and np.isfinite(lse[0]).all()


def test_paged_cache_hands_out_every_page_once():
    c = nkv.PagedCache(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=9, max_rows=200, device="cpu")
    assert c.table.shape == (4, 4) and bool((c.table == -1).all()) and c.free_pages == 9
    c.reserve([1, 64, 65, 0])
    held = c.table[c.table >= 0].tolist()
    assert (c.table >= 0).sum(1).tolist() == [1, 1, 2, 0] and len(set(held)) == 4 and c.free_pages == 5
    c.reserve([1, 10, 129, 0])                                              # what is held stays where it is
    assert c.table[c.table >= 0].tolist()[:4] == held and c.free_pages == 4
    with pytest.raises(MemoryError):
        c.reserve([200, 200, 0, 0])
    with pytest.raises(ValueError):
        c.reserve([257, 0, 0, 0])
    with pytest.raises(ValueError):
        c.reserve([1, 1])
    assert c.free_pages == 4
    c.lens[2:] = 7
    c.release(1)
    assert c.free_pages == 7 and c.lens.tolist() == [0, 0, 0, 0] and (c.table >= 0).sum(1).tolist() == [1, 1, 0, 0]
    c.reserve([256, 64, 0, 0])
    assert c.free_pages == 4 and len(set(c.table[c.table >= 0].tolist())) == 5
    with pytest.raises(nkv.NkvError):
        nkv.PagedCache(1, 1, 80, nkv.DTYPE_BF16, nkv.PAGES_FP4, 1, 64, device="cpu")


def _attention_args():
    """An attention's arguments, on the CPU: good ones but for that, and nothing is launched where a ValueError comes first."""
    c = nkv.PagedCache(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=4, max_rows=64, device="cpu")
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    return dict(q=q, pages=c.pages, n_q_heads=4, n_new=3, scale=1.0, out=torch.zeros(2, 3, 4, 64), lse=torch.zeros(2, 3, 4),
                ws=torch.zeros(1 << 16, dtype=torch.uint8), stream=0)


@pytest.mark.parametrize("bad", [
    dict(out=torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)),             # fp32 rows are twice as long
    dict(out=torch.zeros(2, 3, 4, 64, dtype=torch.float64)), dict(out=torch.zeros(2, 3, 4, 32)), dict(out=torch.zeros(2, 3, 2, 64)),
    dict(out=torch.zeros(3, 2, 4, 64).transpose(0, 1)), dict(out=torch.zeros(2, 3, 4, 128)[..., ::2]),
    dict(lse=torch.zeros(2, 3, 4, dtype=torch.bfloat16)), dict(lse=torch.zeros(2, 3)), dict(lse=torch.zeros(2, 3, 8)[..., ::2]),
    dict(ws=torch.zeros(4, 1 << 16, dtype=torch.uint8)[:, ::2]),          # counted as larger than the piece that it begins
], ids=lambda b: str({k: (tuple(t.shape), t.dtype, t.stride()) for k, t in b.items()}))
def test_binding_refuses_outputs_that_an_attention_would_write_beside(bad):
    with pytest.raises(ValueError, match=next(iter(bad))):
        nkv.pages_attention(**{**_attention_args(), **bad})


@pytest.mark.parametrize("call", [nkv.pages_load, nkv.pages_read], ids=["load", "read"])
@pytest.mark.parametrize("bad", [
    dict(head_off=torch.zeros(5, dtype=torch.int32)),                     # half as long as what is read
    dict(head_off=torch.zeros(4, dtype=torch.int64)), dict(head_off=torch.zeros(10, dtype=torch.int64)[::2]),
    dict(packed_k=torch.zeros(9, 64, dtype=torch.bfloat16)), dict(packed_v=torch.zeros(10, 32, dtype=torch.bfloat16)),
    dict(packed_v=torch.zeros(10, 128, dtype=torch.bfloat16)[:, :64]), dict(packed_k=torch.zeros(64, 10, dtype=torch.bfloat16).T),
    dict(packed_k=torch.zeros(10, 64)),
], ids=lambda b: str({k: (tuple(t.shape), t.dtype, t.stride()) for k, t in b.items()}))
def test_binding_refuses_packed_rows_that_a_call_would_leave(call, bad):
    c = nkv.PagedCache(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=4, max_rows=64, device="cpu")
    rows = torch.zeros(10, 64, dtype=torch.bfloat16)
    good = dict(packed_k=rows, packed_v=rows.clone(), head_off=torch.zeros(5, dtype=torch.int64), rows=10, pages=c.pages, stream=0)
    with pytest.raises(ValueError, match=next(iter(bad))):
        call(**{**good, **bad})


def test_binding_refuses_tensors_that_are_not_where_the_pages_are():
    """A host address handed to a kernel faults the GPU.  (Pages on the CPU and a tensor that says it is on a GPU stand for the two places.)"""
    class OnGpu(torch.Tensor):
        def get_device(self):
            return 0
    c = nkv.PagedCache(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=4, max_rows=64, device="cpu")
    for other in ("pool", "table", "lens"):
        with pytest.raises(ValueError, match="device"):
            nkv.Pages(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, **{**dict(pool=c.pool, table=c.table, lens=c.lens), other: getattr(c, other).to("meta")})
    row = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    append = dict(k=row(2, 3, 2, 64), v=row(2, 3, 2, 64), positions=torch.zeros(2, 3, dtype=torch.int32), rope=torch.zeros(9, 2, 32), q=row(2, 3, 4, 64),
                  q_out=row(2, 3, 4, 64))
    packed = dict(packed_k=row(10, 64), packed_v=row(10, 64), head_off=torch.zeros(5, dtype=torch.int64))
    attend = {x: y for x, y in _attention_args().items() if isinstance(y, torch.Tensor)}
    for call, tensors, rest in ((nkv.pages_append, append, {}), (nkv.pages_load, packed, dict(rows=10)), (nkv.pages_read, packed, dict(rows=10)),
                                (nkv.pages_attention, attend, dict(n_q_heads=4, n_new=3, scale=1.0))):
        for name in tensors:
            with pytest.raises(ValueError, match=f"{name}.*device"):
                call(**{**tensors, **rest, name: tensors[name].as_subclass(OnGpu)}, pages=c.pages, stream=0)
        with pytest.raises(ValueError, match="not on a GPU"):             # all of them in the same wrong place
            call(**tensors, **rest, pages=c.pages, stream=0)


@pytest.mark.parametrize("seq", [-1, -2, 2, 7])
def test_release_refuses_what_is_no_sequence(seq):
    """(-1 would give the last sequence's pages back and leave its lengths: rows on no page.)"""
    c = nkv.PagedCache(2, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=9, max_rows=200, device="cpu")
    c.reserve([1, 1, 70, 70])
    c.lens.copy_(torch.tensor([1, 1, 70, 70]))
    before = c.table.clone()
    with pytest.raises(IndexError):
        c.release(seq)
    assert c.free_pages == 3 and torch.equal(c.table, before) and c.lens.tolist() == [1, 1, 70, 70]
    c.release(1)
    assert c.free_pages == 7 and c.lens.tolist() == [1, 1, 0, 0] and c.table[:2].tolist() == before[:2].tolist() and bool((c.table[2:] == -1).all())


def test_layers_of_a_paged_cache_follow_what_is_reserved_and_released():
    """Sequences (prompt, layer): every layer's table and lengths, where they lie, hold what the owner's do after each step."""
    P, L, H = 3, 2, 2
    c = nkv.PagedCache(P * L, H, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=40, max_rows=200, device="cpu")
    start = torch.arange(P * L * H, dtype=torch.int32) * 5
    c.lens.copy_(start)
    c.reserve(start.tolist())
    layers = c.layers(L)
    where = [(x.table.data_ptr(), x.lens.data_ptr()) for x in layers]

    def in_line():
        for l, x in enumerate(layers):
            assert (x.n_seqs, x.H, x.c.table, x.c.lens) == (P, H, *where[l]) and x.c.pool == c.pool.data_ptr()
            assert torch.equal(x.table, c.table.view(P, L, H, -1)[:, l].reshape(P * H, -1))
            assert (x.table.data_ptr(), x.lens.data_ptr()) == where[l]

    in_line()
    assert torch.equal(c.layer_lens, start.view(P, L, H).transpose(0, 1).reshape(L, P * H))
    c.layer_lens.add_(1)
    assert [x.lens.tolist() for x in layers] == c.layer_lens.tolist()
    c.reserve([130] * (P * L * H))
    in_line()
    c.release(2 * L + 1)                                                    # the last prompt in layer 1
    in_line()
    want = (start.view(P, L, H).transpose(0, 1) + 1).clone()
    want[1, 2] = 0
    assert torch.equal(c.layer_lens.view(L, P, H), want) and c.lens.view(P, L, H)[2, 1].tolist() == [0, 0]
    c.reserve([0] * (P * L - 1) * H + [64] * H)
    in_line()
    assert c.layers(L) == layers and torch.equal(c.layer_lens.view(L, P, H), want)   # the same ones
    for bad in (0, 4, L + 1):
        with pytest.raises(ValueError):
            c.layers(bad)


def test_layers_of_one_prompt_have_lengths_of_their_own():
    c = nkv.PagedCache(3, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, n_pages=12, max_rows=100, device="cpu")
    c.reserve([60] * 6)
    layers = c.layers(3)
    c.layer_lens.add_(1)
    assert c.lens.tolist() == [0] * 6 and [x.lens.tolist() for x in layers] == [[1, 1]] * 3
    c.reserve([70] * 6)
    assert torch.equal(c.layer_table.flatten(0, 1), c.table) and bool((c.table >= 0).all())


def test_attention_refuses_a_scale_that_is_infinite_in_32_bits():
    L, p, n = nkv.lib(), _pages(), C.c_size_t(0)
    assert L.nkv_pages_workspace_bytes(C.byref(p), 8, 1, C.byref(n)) == 0
    for scale in (3e38, -3e38, 1e39, -1e300, float("inf")):                # times log2(e)
        assert L.nkv_pages_attention(FAKE, C.byref(p), 8, 1, scale, FAKE, 0, FAKE, n.value, 0) == nkv.NKV_EINVAL


@pytest.mark.parametrize("fmt,d,dtype", [("fp4", 64, "bf16"), ("fp4", 128, "fp16"), ("fp4", 256, "bf16"), ("16bit", 64, "fp16"), ("16bit", 128, "bf16"), ("16bit", 256, "bf16")])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (3, 2)])
def test_the_bar_of_an_attention_sees_a_lost_piece_of_its_weights(fmt, d, dtype, G, n):
    """The caches and queries of the GPU's test, in 64 bits: weights cut off behind 16 bits, as if a third piece of 8 were lost, leave the bar; plain
    fp32 stays well under it."""
    from pages_util import Cache, attention_bar, from_bits, values_of
    c = Cache(8, 2, d, dtype, fmt, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 700], rows=1.0, seed=d + G)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(c.S, n, 2 * G, d, generator=g).to(c.torch_dtype).double().numpy()
    want, _ = op.attention(q, c.pool, c.table, c.lens, 2, d ** -0.5, d, c.fp4, from_bits(c.torch_dtype))
    cut, f32 = np.zeros_like(want), np.zeros_like(want)
    for u in range(16):
        s, h = divmod(u, 2)
        rows = [op.read_rows(c.pool[c.table[u, j]], d, c.fp4, from_bits(c.torch_dtype)) for j in range((int(c.lens[u]) + 63) // 64)]
        for t in range(n):
            see = int(c.lens[u]) - (n - 1 - t)
            if see < 1:
                continue
            K, V = (np.concatenate([x[i] for x in rows])[:see] for i in range(2))
            heads = slice(h * G, (h + 1) * G)
            z = d ** -0.5 * (q[s, t, heads] @ K.T)
            w = np.exp(z - z.max(-1, keepdims=True))
            short = (w.astype(np.float32).view(np.uint32) & np.uint32(0xffffff00)).view(np.float32).astype(np.float64)
            cut[s, t, heads] = (short / w.sum(-1, keepdims=True)) @ V
            z = np.float32(d ** -0.5) * (q[s, t, heads].astype(np.float32) @ K.astype(np.float32).T)
            w = np.exp(z - z.max(-1, keepdims=True))
            f32[s, t, heads] = (w @ V.astype(np.float32)) / w.sum(-1, keepdims=True)
    bar = attention_bar(np.abs(values_of(c)).max())
    assert np.abs(cut - want).max() > bar
    assert np.abs(f32 - want).max() < bar / 3
