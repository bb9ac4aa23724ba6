"""What attention of prompts' chunks with rules refuses, without a GPU."""
import ctypes as C

import pytest
import torch

import paper_2605_26678_amd as nkv
from test_pages_host import BAD_PAGES, FAKE, _pages


def _rules(**kw):
    r = dict(struct_size=C.sizeof(nkv.nkv_logit_rules), window=5, cap=30.0, slopes=FAKE, prefix=FAKE)
    r.update(kw)
    return C.byref(nkv.nkv_logit_rules(*[r[f] for f, _ in nkv.nkv_logit_rules._fields_]))


def _call(p=None, rules=None, heads=8, new=1, scale=1.0, q=FAKE, out=FAKE, lse=0, ws=FAKE, size=1 << 40):
    return nkv.lib().nkv_pages_prompt_attention(q, C.byref(p or _pages()), rules, heads, new, scale, out, lse, ws, size, 0)


@pytest.mark.parametrize("bad", BAD_PAGES, ids=lambda b: str(b)[:40])
def test_bad_pages(bad):
    (kw, status), n = bad, C.c_size_t(0)
    assert _call(_pages(**kw)) == status
    assert nkv.lib().nkv_pages_prompt_workspace_bytes(C.byref(_pages(**kw)), 8, 1, C.byref(n)) == status


@pytest.mark.parametrize("kw", [dict(struct_size=0), dict(window=-1), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-31), dict(cap=1e39),
                                dict(cap=1e35), dict(slopes=FAKE + 2), dict(prefix=FAKE + 1)], ids=str)
def test_bad_rules(kw):
    assert _call(rules=_rules(**kw)) == nkv.NKV_EINVAL


def test_bad_arguments():
    L, n, p = nkv.lib(), C.c_size_t(0), _pages()
    assert L.nkv_pages_prompt_workspace_bytes(C.byref(p), 8, 1, None) == nkv.NKV_EINVAL
    for heads, new, status in ((2, 1, nkv.NKV_EINVAL), (6, 1, nkv.NKV_EINVAL), (8, 0, nkv.NKV_EINVAL), (8, 1 << 29, nkv.NKV_ESHAPE), (8, 1 << 27, nkv.NKV_ESHAPE)):
        assert L.nkv_pages_prompt_workspace_bytes(C.byref(p), heads, new, C.byref(n)) == status
        assert _call(heads=heads, new=new) == status
    for kw in (dict(q=0), dict(out=0), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(lse=FAKE + 2), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e39)):
        assert _call(**kw) == nkv.NKV_EINVAL
    wide = _pages(max_pages=1000)
    assert L.nkv_pages_prompt_workspace_bytes(C.byref(wide), 8, 1, C.byref(n)) == 0 and n.value > 0
    for ws, size in ((0, n.value), (FAKE + 16, n.value), (FAKE, n.value - 1)):
        assert _call(wide, ws=ws, size=size) == nkv.NKV_EWORKSPACE
    # a short table, or enough columns: no scratch
    assert L.nkv_pages_prompt_workspace_bytes(C.byref(_pages(max_pages=2)), 8, 1, C.byref(n)) == 0 and n.value == 0
    assert L.nkv_pages_prompt_workspace_bytes(C.byref(p), 32, 4096, C.byref(n)) == 0 and n.value == 0


def test_scratch_is_bounded():
    n = C.c_size_t(0)
    for d in (64, 128, 256):
        for S in (1, 3, 64):
            for heads in (4, 32, 128):
                for new in (1, 2, 7, 64, 1000, 5000):
                    assert nkv.lib().nkv_pages_prompt_workspace_bytes(C.byref(_pages(n_seqs=S, d=d, max_pages=1000)), heads, new, C.byref(n)) == 0
                    assert n.value < 80 << 20


def test_windows_beyond_32_bits():
    """A window is an int32 in the header: what is more is refused, not cut off."""
    assert nkv.LogitRules(window=(1 << 31) - 1).c.window == (1 << 31) - 1
    for window in (1 << 31, (1 << 32) + 5, 1 << 62):
        with pytest.raises(ValueError):
            nkv.LogitRules(window=window)


@pytest.mark.parametrize("fmt", [nkv.PAGES_16BIT, nkv.PAGES_FP4])
def test_scratch_is_what_the_header_says(fmt):
    """Few columns: (stretches + units) * columns * (d + 4) * 4 bytes and 16 a unit, or none; more of them: 33 MiB at most."""
    n, needed = C.c_size_t(0), set()
    for d, stretches in ((64, 4096), (96, 3072), (128, 3072), (192, 2048), (256, 2048)):
        for S in (1, 2, 31, 256, 1024):
            for H in (1, 8):
                for width in (1, 4, 5, 20, 21, 32, 33, 100, 1000):
                    for cols in (1, 5, 16, 17, 32, 33, 64, 257, 1000, 20000):
                        assert nkv.lib().nkv_pages_prompt_workspace_bytes(C.byref(_pages(n_seqs=S, H=H, d=d, format=fmt, max_pages=width)), H * cols, 1, C.byref(n)) == 0
                        units, few = S * H, cols <= 16 and width > 20 if fmt == nkv.PAGES_16BIT else cols <= (32 if width > 32 else 16)
                        parts = min(stretches, 4 * ((units * width + 3) // 4)) + units
                        bound = parts * cols * (d + 4) * 4 + (16 * units + 255) // 256 * 256
                        what = f"{units} units of {width} pages, {cols} columns of {d} dims"
                        assert n.value in (0, bound) if few else n.value <= 33 << 20, what
                        needed.add((few, n.value > 0))
    assert len(needed) == 4
    if fmt == nkv.PAGES_FP4:                                                # (the header's figures)
        for S, mib in ((1, 50), (256, 83), (1024, 182)):
            assert nkv.lib().nkv_pages_prompt_workspace_bytes(C.byref(_pages(n_seqs=S, H=8, d=128, format=fmt, max_pages=1000)), 256, 1, C.byref(n)) == 0
            assert round(n.value / 2 ** 20) == mib


def test_binding_refuses():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    table, lens = z(2, 3, dt=torch.int32), z(2, dt=torch.int32)
    pages = nkv.Pages(1, 2, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, z(4, nkv.page_bytes(64, nkv.DTYPE_BF16, nkv.PAGES_FP4), dt=torch.uint8), table, lens)
    f, i = z(4, dt=torch.float32), z(1, dt=torch.int32)
    for bad in (dict(slopes=f.double()), dict(slopes=z(2, 2, dt=torch.float32)), dict(slopes=z(8, dt=torch.float32)[::2]), dict(prefix=i.long()), dict(cap=-1.0),
                dict(cap=float("nan")), dict(window=-1)):
        with pytest.raises(ValueError):
            nkv.LogitRules(**bad)
    q = z(1, 3, 4, 64)
    good = dict(q=q, pages=pages, n_q_heads=4, n_new=3, scale=1.0, out=torch.zeros_like(q), lse=z(1, 3, 4, dt=torch.float32), ws=z(1 << 20, dt=torch.uint8),
                rules=nkv.LogitRules(1.0, 2, f, i))
    for bad in (dict(q=q.half()), dict(q=q[:, :2]), dict(out=q.float()), dict(out=z(1, 3, 4, 128)[..., ::2]), dict(lse=z(1, 3, 4)), dict(lse=z(1, 3, 3, dt=torch.float32)),
                dict(ws=z(8, 8, dt=torch.uint8)[:, ::2]), dict(rules=nkv.LogitRules(slopes=f[:3])), dict(rules=nkv.LogitRules(prefix=i[:0])), dict()):
        with pytest.raises(ValueError):
            nkv.pages_prompt_attention(**{**good, **bad}, stream=0)
