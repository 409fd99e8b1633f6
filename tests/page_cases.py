"""Caches in pages for tests: pools, tables and windows, and plain 64-bit forms
of the operators that work on them."""
import math

import torch

from paper_2405_14105_amd import dsi

KIND = {torch.float32: dsi.DSI_F32, torch.bfloat16: dsi.DSI_BF16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


class Step:
    """Windows with `past` cached positions and `rows` new ones each, in a pool of
    shuffled pages.  What no row of the step may read is NaN."""

    def __init__(self, rows, past, hkv, hd, kv, page, reach=0, seed=0, before=0, behind=0, spare=2):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.past, self.hkv, self.hd, self.page, self.reach = rows, past, hkv, hd, page, reach
        self.before, self.n = before, before + sum(rows) + behind
        B = len(rows)
        need = [max(1, -(-(p + r) // page)) for p, r in zip(past, rows)]
        order = torch.randperm(sum(need) + spare, generator=g)
        self.most = max(need) + 1
        self.table = torch.full((B, self.most), -7, dtype=torch.int32)
        self.K = [torch.randn((p + r, hkv, hd), generator=g).to(kv) for p, r in zip(past, rows)]
        self.V = [torch.randn((p + r, hkv, hd), generator=g).to(kv) for p, r in zip(past, rows)]
        pages = len(order)
        self.k = torch.full((pages, hkv, page // 32, hd // 32, 32, 32), math.nan).to(kv)
        self.v = torch.full((pages, hkv, page // 32, hd, 32), math.nan).to(kv)
        at = 0
        for b in range(B):
            low = max(0, past[b] - reach + 1) if reach else 0
            for e in range(need[b]):
                page_id = int(order[at + e])
                if (e + 1) * page > low and e * page < past[b] + rows[b]:
                    self.table[b, e] = page_id
                lo, hi = max(e * page, low), min((e + 1) * page, past[b] + rows[b])
                if hi > lo:
                    p = torch.arange(lo, hi)
                    place = p - e * page
                    self.k[page_id][:, place // 32, :, place % 32] = self.K[b][lo:hi].view(hi - lo, hkv, hd // 32, 32)
                    self.v[page_id][:, place // 32, :, place % 32] = self.V[b][lo:hi]
            at += need[b]
        self.row0 = torch.tensor([before + sum(rows[:b]) for b in range(B + 1)], dtype=torch.int32)
        self.len = torch.tensor(past, dtype=torch.int32)

    def to(self, dev):
        for name in ("table", "k", "v", "row0", "len"):
            setattr(self, name, getattr(self, name).to(dev))
        return self

    def pages(self, **change):
        a = dict(n_kv_heads=self.hkv, head_dim=self.hd, kvdtype=KIND[self.k.dtype], n_pages=self.k.shape[0], page_size=self.page, d_k=self.k,
                 d_v=self.v, n_windows=len(self.rows), max_pages=self.most, d_table=self.table, d_len=self.len, d_row0=self.row0)
        return dsi.make_pages(**{**a, **change})

    def keys(self, b):
        """K, V [positions][hkv][hd] of a window as the pool holds them (page by page)."""
        n = self.past[b] + self.rows[b]
        p = torch.arange(n)
        page = self.table[b].long().cpu()[p // self.page]
        place = p % self.page
        k, v = self.k.cpu(), self.v.cpu()
        return k[page, :, place // 32, :, place % 32].reshape(n, self.hkv, self.hd), v[page, :, place // 32, :, place % 32]


def attend64(step, q, hq, scale=0.0):
    """Outputs of every row in 64 bits (NaN outside the windows), and for each the sum of p |v| and the largest sum |q k| scale."""
    hkv, hd = step.hkv, step.hd
    scale = scale or 1 / math.sqrt(hd)
    out = torch.full((step.n, hq, hd), math.nan, dtype=torch.float64)
    mass, reachable = torch.zeros_like(out), torch.ones((step.n, hq, 1), dtype=torch.float64)
    r0 = step.before
    for b, n in enumerate(step.rows):
        K, V = step.K[b].double(), step.V[b].double()
        for i in range(n):
            pos = step.past[b] + i
            lo = max(0, pos - step.reach + 1) if step.reach else 0
            for h in range(hq):
                x = q[r0 + i, h].double()
                k, v = K[lo:pos + 1, h // (hq // hkv)], V[lo:pos + 1, h // (hq // hkv)]
                p = torch.softmax(k @ x * scale, 0)
                out[r0 + i, h] = p @ v
                mass[r0 + i, h] = p @ v.abs()
                reachable[r0 + i, h] = (k.abs() @ x.abs()).max() * scale
        r0 += n
    return out, mass, reachable
