"""Inputs of the paged cache's tests: pools, tables and rows, made on the CPU."""
import numpy as np
import torch

from oracle import pages as op
import paper_2605_26678_amd as nkv

DTYPES = {"bf16": (torch.bfloat16, nkv.DTYPE_BF16), "fp16": (torch.float16, nkv.DTYPE_F16)}
FORMATS = {"fp4": nkv.PAGES_FP4, "16bit": nkv.PAGES_16BIT}


def to_bits(dtype):
    """fp64 numpy -> bits of the type, through fp32 as the library rounds."""
    return lambda x: torch.from_numpy(np.asarray(x, np.float32)).to(dtype).view(torch.int16).numpy().view(np.uint16)


def from_bits(dtype):
    return lambda w: torch.from_numpy(np.ascontiguousarray(w).view(np.int16)).view(dtype).double().numpy()


def attention_bar(v_max: float) -> float:
    """What an attention's output may be off by at logits of a few: sums in fp32 of d products and of some hundred weighted values leave up to a third of it (plain
    fp32 on the CPU over the tests' caches: 0.02 to 0.17 of it), and weights that lose their last 8 of 24 bits come out at 1.2 to 4 times it."""
    return 2e-6 * max(1.0, v_max)


def values_of(c):
    """V rows of all units, fp64, one below the other."""
    rows = [op.read_rows(c.pool[c.table[u, j]], c.d, c.fp4, from_bits(c.torch_dtype))[1][:min(64, int(n) - 64 * j)]
            for u, n in enumerate(c.lens) for j in range((int(n) + 63) // 64)]
    return np.concatenate(rows)


class Cache:
    """A pool of pages for units of the given lengths (uint8 numpy), every unit's pages anywhere; the rows behind a unit's last
    one, and pages that nobody has, are all ones (NaN in either format).  Unused table entries are -1."""

    def __init__(self, n_seqs, H, d, dtype, fmt, lens, width=None, seed=0, rows=None):
        self.S, self.H, self.d, self.fp4 = n_seqs, H, d, fmt == "fp4"
        self.torch_dtype, self.dtype = DTYPES[dtype]
        self.fmt = FORMATS[fmt]
        self.lens = np.asarray(lens, np.int32).reshape(n_seqs * H)
        r = np.random.RandomState(seed)
        need = (np.maximum(self.lens, 0) + 63) // 64
        self.width = int(width or max(1, need.max()))
        n_pages = int(need.sum()) + 2
        order = r.permutation(n_pages)
        self.table = np.full((n_seqs * H, self.width), -1, np.int32)
        at = 0
        for u, n in enumerate(need):
            self.table[u, :n] = order[at:at + n]
            at += n
        self.pool = np.full((n_pages, op.page_bytes(d, self.fp4)), 255, np.uint8)
        if rows is not None:
            self.fill(rows, seed)

    def fill(self, spread, seed):
        """Random rows everywhere.  (All pages at once: the definition row by row would take long.)"""
        g = torch.Generator().manual_seed(seed)
        d = self.d
        for u in range(self.S * self.H):
            n = int(self.lens[u])
            mean = torch.randn(2, 1, d, generator=g) * 0.7
            for j in range((n + 63) // 64):
                page = self.pool[self.table[u, j]]
                m = min(64, n - 64 * j)
                x = (torch.randn(2, 64, d, generator=g) * spread + mean)[:, :m].to(self.torch_dtype)
                if not self.fp4:
                    w = page.view(np.uint16).reshape(2, 64, d)
                    w[:, :m] = x.view(torch.int16).numpy().view(np.uint16)
                    continue
                k, v, ks, vs = op.places(d)
                for y, c, s in ((x[0], k, ks), (x[1], v, vs)):
                    # any codes and scales are a valid cache
                    code = torch.randint(0, 16, (m, d), generator=g).numpy().astype(np.uint8)
                    page[c[:m, 0::2]] = code[:, 0::2] | code[:, 1::2] << 4
                    page[s[:m]] = torch.randint(122, 127, (m, d // 32), generator=g).numpy().astype(np.uint8)

    def on(self, dev):
        self.d_pool, self.d_table, self.d_lens = (torch.from_numpy(x.copy()).to(dev) for x in (self.pool, self.table, self.lens))
        return nkv.Pages(self.S, self.H, self.d, self.dtype, self.fmt, self.d_pool, self.d_table, self.d_lens)
