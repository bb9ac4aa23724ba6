"""Copies of pages and compaction on the GPU, bit by bit against oracle/pages.py's layout."""
import numpy as np
import pytest
import torch

from oracle import pages as op
import paper_2605_26678_amd as nkv
from pages_util import Cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [(d, dt, fmt) for d in (64, 96, 128, 192, 256) for dt, fmt in (("bf16", "fp4"), ("fp16", "16bit"))]


def _i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


@pytest.mark.parametrize("d,dtype,fmt", KINDS)
def test_copy(d, dtype, fmt):
    c = Cache(2, 3, d, dtype, fmt, [0, 1, 64, 65, 300, 130], seed=d, rows=1.0)
    pages, n = c.on(DEV), c.pool.shape[0]
    src, dst = [0, 3, 5, -1, 2, n, 7, 4], [9, 8, 5, 6, n, 1, -5, 10]      # (a page to itself, and numbers that are none)
    for k in (0, 1, len(src)):
        pages = c.on(DEV)
        nkv.pages_copy(_i32(src[:k]), _i32(dst[:k]), pages)
        want = c.pool.copy()
        for a, b in zip(src[:k], dst[:k]):
            if 0 <= a < n and 0 <= b < n:
                want[b] = c.pool[a]
        assert np.array_equal(c.d_pool.cpu().numpy(), want), k
        assert np.array_equal(c.d_table.cpu().numpy(), c.table) and np.array_equal(c.d_lens.cpu().numpy(), c.lens)


def test_copy_of_many_pages():
    pool = torch.randint(0, 256, (5001, nkv.page_bytes(64, nkv.DTYPE_BF16, nkv.PAGES_FP4)), dtype=torch.uint8, device=DEV)
    t = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
    pages = nkv.Pages(1, 1, 64, nkv.DTYPE_BF16, nkv.PAGES_FP4, pool, t, t[0])
    order = torch.randperm(5000, generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
    want = pool.clone()
    want[order[:2500].long()] = pool[order[2500:].long()]
    nkv.pages_copy(order[2500:], order[:2500], pages)
    assert torch.equal(pool, want)


def _bytes_of_row(page, row, d, fp4):
    """Everything that belongs to a row."""
    if not fp4:
        w = page.reshape(2, 64, 2 * d)
        return np.concatenate([w[0, row], w[1, row]])
    k, v, ks, vs = op.places(d)
    return np.concatenate([page[k[row, 0::2]], page[v[row, 0::2]], page[ks[row]], page[vs[row]]])


def _zero_row(d, fp4):
    return np.concatenate([np.zeros(d, np.uint8), np.ones(d // 16, np.uint8)]) if fp4 else np.zeros(4 * d, np.uint8)


def _check_compact(c, kept, to_len, other_pool=False, rows=None, to_width=None, stream=None):
    """kept: numbers per unit; to_len: pages' worth of rows of the new table (others -1)."""
    pages = c.on(DEV)
    units, n_old = c.S * c.H, c.pool.shape[0]
    need = [(len(k) + 63) // 64 for k in kept]
    new_pool = np.full((n_old + sum(need) + 1, c.pool.shape[1]), 77, np.uint8)
    width = to_width or max(1, max(need))
    table, at = np.full((units, width), -1, np.int32), n_old if not other_pool else 0
    for u, m in enumerate(need):
        m = min(m, to_len if to_len is not None else m, width)
        table[u, :m] = np.arange(at, at + m)[::-1]
        at += m
    if not other_pool:
        new_pool[:n_old] = c.pool
    off = np.concatenate([[0], np.cumsum([len(k) for k in kept])]).astype(np.int64)
    idx = np.concatenate([np.asarray(k, np.int64) for k in kept] + [np.zeros(0, np.int64)]).astype(np.int32)
    rows = len(idx) if rows is None else rows
    d_new = torch.from_numpy(new_pool.copy()).to(DEV)
    old = pages if other_pool else nkv.Pages(c.S, c.H, c.d, c.dtype, c.fmt, d_new, c.d_table, c.d_lens)
    to = nkv.Pages(c.S, c.H, c.d, c.dtype, c.fmt, d_new, torch.from_numpy(table).to(DEV), torch.full((units,), -9, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    nkv.pages_compact(_i32(idx[:rows]) if rows else _i32([0]), torch.from_numpy(off).to(DEV), rows, old, to, stream=stream)
    torch.cuda.synchronize()
    got = d_new.cpu().numpy()
    want = new_pool.copy()
    for u in range(units):
        for j, i in enumerate(kept[u]):
            if off[u] + j >= rows or j // 64 >= width or table[u, j // 64] < 0:
                continue
            p = int(c.table[u, i // 64]) if 0 <= i < min(int(c.lens[u]), 64 * c.width) else -1
            src = _bytes_of_row(c.pool[p], i % 64, c.d, c.fp4) if 0 <= p < n_old else _zero_row(c.d, c.fp4)
            page = want[table[u, j // 64]]
            if c.fp4:
                k, v, ks, vs = op.places(c.d)
                r = j % 64
                for where, part in zip((k[r, 0::2], v[r, 0::2], ks[r], vs[r]), np.split(src, np.cumsum([c.d // 2, c.d // 2, c.d // 32]))):
                    page[where] = part
            else:
                w = page.reshape(2, 64, 2 * c.d)
                w[0, j % 64], w[1, j % 64] = src[:2 * c.d], src[2 * c.d:]
    bad = np.argwhere(got != want)
    assert bad.size == 0, f"{len(bad)} bytes, the first at {bad[0]}"


def _some(c, share, seed):
    r = np.random.RandomState(seed)
    return [np.flatnonzero(r.rand(max(0, int(n))) < share) for n in c.lens]


@pytest.mark.parametrize("d,dtype,fmt", KINDS)
@pytest.mark.parametrize("share", [0.0, 0.4, 1.0])
def test_compact(d, dtype, fmt, share):
    c = Cache(2, 4, d, dtype, fmt, [0, 1, 63, 64, 65, 129, 700, 0], seed=d, rows=1.0)
    _check_compact(c, _some(c, share, 1), None)
    _check_compact(c, _some(c, share, 2), None, other_pool=True)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_compact_many_units(fmt):
    r = np.random.RandomState(4)
    c = Cache(12, 7, 64, "bf16", fmt, r.randint(0, 200, 84), seed=5, rows=1.0)      # more units than a wavefront has lanes
    _check_compact(c, _some(c, 0.5, 3), None)


@pytest.mark.parametrize("fmt", ["fp4", "16bit"])
def test_compact_what_is_not_there(fmt):
    c = Cache(1, 3, 128, "bf16", fmt, [200, 100, 150], seed=6, rows=1.0)
    c.table[0, 1] = -1                                     # a page that is none, and one beyond the pool
    c.table[2, 0] = 1 << 20
    kept = [np.arange(0, 200, 2), np.array([5, 5, 3, 99, 100, -1, 1 << 30, 0]), np.arange(149, -1, -1)]
    _check_compact(c, kept, None)
    _check_compact(c, kept, 1)                             # only the first new page of a unit is one
    _check_compact(c, kept, None, to_width=1)
    _check_compact(c, kept, None, rows=120)                # head_off beyond what kept_idx holds
    _check_compact(c, kept, None, rows=0)
    c.lens[1] = 4000                                       # beyond the table
    _check_compact(c, kept, None)
    c.lens[1] = -4
    _check_compact(c, kept, None)


def test_compact_on_a_stream_and_in_a_graph():
    c = Cache(1, 2, 128, "bf16", "fp4", [300, 200], seed=7, rows=1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _check_compact(c, _some(c, 0.5, 8), None, stream=side)
    pages = c.on(DEV)
    kept = _some(c, 0.5, 9)
    off = torch.tensor([0, len(kept[0]), len(kept[0]) + len(kept[1])], device=DEV)
    idx, rows = _i32(np.concatenate(kept)), len(kept[0]) + len(kept[1])
    pool = torch.zeros(20, c.pool.shape[1], dtype=torch.uint8, device=DEV)
    table = torch.arange(20, dtype=torch.int32, device=DEV).view(2, 10)
    to = nkv.Pages(1, 2, 128, c.dtype, c.fmt, pool, table, c.d_lens)
    src, dst = _i32([0, 1]), _i32([18, 19])
    nkv.pages_compact(idx, off, rows, pages, to)
    nkv.pages_copy(src, dst, to)
    want = pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nkv.pages_compact(idx, off, rows, pages, to)
        nkv.pages_copy(src, dst, to)
    for _ in range(4):
        pool.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want)
