"""A small paged cache on the host and its operators in 64 bits, from their definition, for the paged tests."""
import numpy as np
import torch

from paper_2609_32663_gb300 import dkv

HEAD = 128


class Cache:
    """Slabs of given lengths (int [L, B, Hkv]) on pages in random order. Pool rows that no slab holds are NaN."""

    def __init__(self, lens, page, spare=3, wider=2, dtype=torch.bfloat16, seed=0, H=None):
        lens = np.asarray(lens, np.int64)
        self.L, self.B, self.Hkv = lens.shape
        self.H = H or self.Hkv
        self.P, self.lens, self.dtype = page, lens.reshape(-1).copy(), dtype
        r = np.random.default_rng(seed)
        pages = -(-self.lens // page)
        total = int(pages.sum())
        order = r.permutation(total + spare).astype(np.int32)
        self.table = np.full((self.lens.size, int(pages.max(initial=0)) + wider), 0x7f7f7f7f, np.int32)
        self.table[np.arange(self.table.shape[1])[None] < pages[:, None]] = order[:total]
        self.free = np.full(total + spare, -7, np.int32)
        self.free[:spare] = order[total:]
        self.count = spare
        gen = torch.Generator().manual_seed(seed)
        rows = (total + spare) * page
        self.Kp = torch.full((rows, HEAD), float("nan"), dtype=dtype)
        self.Vp = self.Kp.clone()
        for h in range(self.lens.size):
            at = self.rows(h)
            self.Kp[at] = torch.randn((at.size, HEAD), generator=gen).to(dtype)
            self.Vp[at] = torch.randn((at.size, HEAD), generator=gen).to(dtype)
        self.pages = dkv.Pages(L=self.L, B=self.B, H=self.H, H_kv=self.Hkv, page_rows=page, num_pages=total + spare,
                               max_pages=self.table.shape[1])

    def rows(self, h, first=0, last=None):
        """Pool rows of rows [first, last) of slab h."""
        r = np.arange(first, self.lens[h] if last is None else last)
        return self.table[h][r // self.P].astype(np.int64) * self.P + r % self.P


def attention(cache, layer, q, k_new, v_new, cu, causal, scale=None):
    """(out, sum_r w_r |v_r|, Kp, Vp) in 64 bits: what dkv_chunk_attn gives for host tensors; rows behind the last
    sequence are NaN in out."""
    Kp, Vp = cache.Kp.double().clone(), cache.Vp.double().clone()
    out = torch.full(q.shape, float("nan"), dtype=torch.float64)
    size = torch.zeros(q.shape, dtype=torch.float64)
    G = cache.H // cache.Hkv
    scale = HEAD ** -0.5 if scale is None else scale
    for b in range(cache.B):
        t0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        for g in range(cache.Hkv):
            h = (layer * cache.B + b) * cache.Hkv + g
            m = int(cache.lens[h])
            at = cache.rows(h)
            if k_new is not None and n:
                Kp[at[m - n:]] = k_new[t0:t0 + n, g].double()
                Vp[at[m - n:]] = v_new[t0:t0 + n, g].double()
            K, V = Kp[at], Vp[at]
            for i in range(n):
                sees = max(0, m - n + i + 1) if causal else m
                for j in range(g * G, (g + 1) * G):
                    if sees == 0:
                        out[t0 + i, j] = 0
                        continue
                    w = torch.softmax(K[:sees] @ q[t0 + i, j].double() * scale, 0)
                    out[t0 + i, j] = w @ V[:sees]
                    size[t0 + i, j] = w @ V[:sees].abs()
    return out, size, Kp, Vp


def assert_attention(got, want, size, dtype, what=""):
    """Each output is rounded once (half a step of |o|), and so is each softmax weight (half a step of sum w|v| at
    most); scores are 32-bit sums of 128 products, |error| <= 128 2^-24 sum|q k| scale < 2e-4 for the standard normal
    inputs here (sum |q k| scale < 25), which moves a weight by twice that."""
    u = torch.finfo(dtype).eps / 2
    got = got.double().cpu()
    bound = u * (want.abs() + size) + 4e-4 * size + 1e-30
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)]), what
    err = ((got - want).abs() / bound)[finite]
    assert err.numel() == 0 or float(err.max()) <= 1, f"{what}: {float(err.max()):.3g} times the bound"


def tables_after(cache, n_rows, release=False):
    """Tables, free list and counts after dkv_page_tables with n_rows[h] new rows (or dkv_page_release of the slabs with
    n_rows[h] != 0): (table, free, count, len)."""
    P, table, free, ln = cache.P, cache.table.copy(), cache.free.copy(), cache.lens.copy()
    count = cache.count
    for h, n in enumerate(np.asarray(n_rows).reshape(-1)):
        had = -(-int(ln[h]) // P)
        if release:
            if n:
                free[count:count + had] = table[h, :had]
                count += had
                ln[h] = 0
            continue
        for p in range(had, -(-int(ln[h] + n) // P)):
            count -= 1
            table[h, p] = free[count]
        ln[h] += n
    return table, free, count, ln
