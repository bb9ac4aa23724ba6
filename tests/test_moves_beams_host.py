"""What copies, compaction and beam selection refuse, without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2605_26678_amd as nkv
from test_pages_host import BAD_PAGES, FAKE, _pages


@pytest.mark.parametrize("bad", BAD_PAGES, ids=lambda b: str(b)[:40])
def test_bad_pages(bad):
    L, (kw, status) = nkv.lib(), bad
    p, good = _pages(**kw), _pages()
    assert L.nkv_pages_copy(FAKE, FAKE, 1, C.byref(p), 0) == status
    assert L.nkv_pages_compact(FAKE, FAKE, 1, C.byref(p), C.byref(good), 0) == status
    assert L.nkv_pages_compact(FAKE, FAKE, 1, C.byref(good), C.byref(p), 0) == status


def test_copy_and_compact_refuse():
    L, p = nkv.lib(), _pages()
    for src, dst, n, status in ((0, FAKE, 1, nkv.NKV_EINVAL), (FAKE, 0, 1, nkv.NKV_EINVAL), (FAKE + 2, FAKE, 1, nkv.NKV_EINVAL), (FAKE, FAKE, -1, nkv.NKV_EINVAL),
                                (FAKE, FAKE, 1 << 22, nkv.NKV_ESHAPE), (0, 0, 0, nkv.NKV_OK)):
        assert L.nkv_pages_copy(src, dst, n, C.byref(p), 0) == status
    for kept, off, rows, status in ((0, FAKE, 1, nkv.NKV_EINVAL), (FAKE, 0, 1, nkv.NKV_EINVAL), (FAKE + 1, FAKE, 1, nkv.NKV_EINVAL), (FAKE, FAKE + 4, 1, nkv.NKV_EINVAL),
                                    (FAKE, FAKE, -1, nkv.NKV_EINVAL), (FAKE, FAKE, 1 << 40, nkv.NKV_ESHAPE), (0, FAKE, 0, nkv.NKV_OK)):
        assert L.nkv_pages_compact(kept, off, rows, C.byref(p), C.byref(_pages(table=2 * FAKE)), 0) == status
    assert L.nkv_pages_compact(FAKE, FAKE, 0, C.byref(p), C.byref(p), 0) == nkv.NKV_EINVAL                  # onto itself
    for other in (dict(n_seqs=1), dict(H=2), dict(d=64), dict(dtype=nkv.DTYPE_F16), dict(format=nkv.PAGES_16BIT)):
        assert L.nkv_pages_compact(FAKE, FAKE, 1, C.byref(p), C.byref(_pages(**other)), 0) == nkv.NKV_ESHAPE


def _beams(**kw):
    b = dict(struct_size=C.sizeof(nkv.nkv_beams), n_prompts=2, n_beams=4, vocab=1000, n_out=8, dtype=nkv.DTYPE_BF16, strides=(C.c_int64 * 2)(4000, 1000),
             logits=FAKE, scores=FAKE)
    b.update(kw)
    return nkv.nkv_beams(*[b[f] for f, _ in nkv.nkv_beams._fields_])


@pytest.mark.parametrize("kw,status", [
    (dict(struct_size=1), nkv.NKV_EINVAL), (dict(n_prompts=0), nkv.NKV_ESHAPE), (dict(n_beams=0), nkv.NKV_ESHAPE), (dict(vocab=0), nkv.NKV_ESHAPE), (dict(n_beams=1025), nkv.NKV_ESHAPE),
    (dict(n_out=0), nkv.NKV_EINVAL), (dict(n_out=65), nkv.NKV_EINVAL), (dict(dtype=nkv.DTYPE_F8_E4M3), nkv.NKV_EUNSUPPORTED), (dict(dtype=9), nkv.NKV_EINVAL),
    (dict(dtype=-1), nkv.NKV_EINVAL), (dict(logits=0), nkv.NKV_EINVAL), (dict(scores=0), nkv.NKV_EINVAL), (dict(logits=FAKE + 1), nkv.NKV_EINVAL),
    (dict(logits=FAKE + 2, dtype=nkv.DTYPE_F32), nkv.NKV_EINVAL), (dict(scores=FAKE + 2), nkv.NKV_EINVAL), (dict(vocab=(1 << 30) + 1), nkv.NKV_ESHAPE),
    (dict(vocab=1 << 30), nkv.NKV_ESHAPE), (dict(n_prompts=1 << 24, n_beams=1, vocab=1), nkv.NKV_ESHAPE), (dict(n_prompts=1 << 23, n_beams=2, vocab=1), nkv.NKV_ESHAPE),
], ids=str)
def test_beams_refuse(kw, status):
    L, n = nkv.lib(), C.c_size_t(0)
    assert L.nkv_beam_workspace_bytes(C.byref(_beams(**kw)), C.byref(n)) == status
    assert L.nkv_beam_select(C.byref(_beams(**kw)), FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == status


def test_beams_of_more_prompts_than_one_launch_joins():
    """A workgroup of 1024 threads a prompt, and fewer than 2^32 threads."""
    L, n = nkv.lib(), C.c_size_t(0)
    for prompts, status in (((1 << 22) - 1, nkv.NKV_OK), (1 << 22, nkv.NKV_ESHAPE), ((1 << 24) - 1, nkv.NKV_ESHAPE)):
        b = _beams(n_prompts=prompts, n_beams=1, vocab=5, n_out=4)
        assert L.nkv_beam_workspace_bytes(C.byref(b), C.byref(n)) == status
        if status:
            assert L.nkv_beam_select(C.byref(b), FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == status


def test_beams_refuse_outputs_and_scratch():
    L, n, b = nkv.lib(), C.c_size_t(0), _beams()
    assert L.nkv_beam_workspace_bytes(C.byref(b), None) == nkv.NKV_EINVAL and L.nkv_beam_workspace_bytes(None, C.byref(n)) == nkv.NKV_EINVAL
    assert L.nkv_beam_workspace_bytes(C.byref(b), C.byref(n)) == 0 and n.value == nkv.beam_workspace_bytes(2, 4, 1000, 8)
    for outs in ((0, FAKE, FAKE), (FAKE, 0, FAKE), (FAKE, FAKE, 0), (FAKE + 2, FAKE, FAKE), (FAKE, FAKE + 1, FAKE), (FAKE, FAKE, FAKE + 3)):
        assert L.nkv_beam_select(C.byref(b), *outs, FAKE, n.value, 0) == nkv.NKV_EINVAL
    for ws, size in ((0, n.value), (FAKE + 16, n.value), (FAKE, n.value - 1)):
        assert L.nkv_beam_select(C.byref(b), FAKE, FAKE, FAKE, ws, size, 0) == nkv.NKV_EWORKSPACE


def test_binding_refuses():
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)  # noqa: E731
    good = dict(logits=z(2, 3, 50), scores=z(2, 3), out_scores=z(2, 4), out_beams=z(2, 4, dt=torch.int32), out_tokens=z(2, 4, dt=torch.int32),
                ws=z(10000, dt=torch.uint8))
    for bad in (dict(logits=z(2, 3, 50, dt=torch.float64)), dict(logits=z(3, 50)), dict(logits=z(2, 3, 100)[..., ::2]), dict(scores=z(2, 4)),
                dict(scores=z(2, 3, dt=torch.float64)), dict(scores=z(3, 2).T), dict(out_scores=z(3, 4)), dict(out_scores=z(8)), dict(out_beams=z(2, 4)),
                dict(out_tokens=z(2, 5, dt=torch.int32)), dict(ws=z(100, 100, dt=torch.uint8)[:, ::2]), dict()):        # (the last: on the CPU)
        with pytest.raises(ValueError):
            nkv.beam_select(**{**good, **bad}, stream=0)
    table, lens = z(2, 3, dt=torch.int32), z(2, dt=torch.int32)
    pages = nkv.Pages(1, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, z(4, nkv.page_bytes(64, nkv.DTYPE_BF16, nkv.PAGES_FP4), dt=torch.uint8), table, lens)
    i, off = z(5, dt=torch.int32), z(3, dt=torch.int64)
    for src, dst in ((i, i[:4]), (i.long(), i.long()), (i, i.long()), (z(10, dt=torch.int32)[::2], i), (i, i)):
        with pytest.raises(ValueError):
            nkv.pages_copy(src, dst, pages, stream=0)
    for kept, o, rows in ((i, off, 6), (i.long(), off, 5), (i, off.int(), 5), (i, off[:2], 5), (i, off, 5)):
        with pytest.raises(ValueError):
            nkv.pages_compact(kept, o, rows, pages, pages, stream=0)
