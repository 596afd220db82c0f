"""Batches, pools and calls shared by the tests of the paged cache."""
from __future__ import annotations

import numpy as np

from oracle import paged

BF16_HALF_STEP = 2.0 ** -8     # relative rounding of a bf16 value
E4M3_HALF_STEP = 2.0 ** -4     # relative rounding of an e4m3 value (normal numbers)


def bf16(x):
    """fp64 values of the array rounded to bf16."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().float().numpy().astype(np.float64)


class Batch:
    """Sequences with `rows` new tokens and `kv` cached ones, pages dealt out at random; the pool's unused slots and pages hold NaN."""

    def __init__(self, rows, kv, kv_heads, d, page_size=16, e4m3=False, seed=0, extra_rows=0, extra_pages=2, extra_width=1, scale=1.0):
        rng = np.random.default_rng(seed)
        self.rows, self.kv, self.kv_heads, self.d, self.size, self.e4m3 = list(rows), list(kv), kv_heads, d, page_size, e4m3
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int64)
        self.T = int(self.cu[-1]) + extra_rows
        counts = [-(-n // page_size) for n in kv]
        self.num_pages = sum(counts) + extra_pages
        order = rng.permutation(self.num_pages)
        width = max(counts, default=0) + extra_width
        self.table = np.full((len(kv), width), -1, dtype=np.int64)     # (entries behind the last page are not read)
        at = 0
        for i, n in enumerate(counts):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.row = d if not e4m3 else (d + 15) // 16 * 16
        shape = (self.num_pages, kv_heads, page_size, d)
        self.k, self.v = np.full(shape, np.nan), np.full(shape, np.nan)
        self.k_code, self.v_code = (np.full(shape[:3] + (self.row,), 127, dtype=np.uint8) for _ in range(2))
        self.k_byte, self.v_byte = (np.full(shape[:3], 255, dtype=np.uint8) for _ in range(2))
        for s, n in enumerate(kv):
            for which in "kv":
                x = bf16(rng.standard_normal((n, kv_heads, d)) * scale * 2.0 ** rng.integers(-1, 2, (n, kv_heads, 1)))
                pool, codes, bytes_ = getattr(self, which), getattr(self, which + "_code"), getattr(self, which + "_byte")
                if e4m3:
                    c, b = paged.quantise(x)
                    x = paged.dequantise(c, b)
                for p in range(n):
                    page, slot = self.table[s, p // page_size], p % page_size
                    pool[page, :, slot] = x[p]
                    if e4m3:
                        codes[page, :, slot, :d], codes[page, :, slot, d:], bytes_[page, :, slot] = c[p], 0, b[p]
        self.rng = rng

    def device(self, A, interleaved=False):
        """(KVCache, KVBatch) on the GPU; interleaved: k and v pages alternate in one allocation."""
        import torch
        cuda = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()
        if self.e4m3:
            pools = [torch.from_numpy(c).cuda().view(torch.float8_e4m3fn) for c in (self.k_code, self.v_code)]
            scales = [torch.from_numpy(b).cuda() for b in (self.k_byte, self.v_byte)]
        else:
            pools, scales = [cuda(x, torch.bfloat16) for x in (self.k, self.v)], [None, None]
        if interleaved:
            both = torch.stack([p.view(torch.uint8) for p in pools], dim=1)
            pools = [both[:, i].view(pools[0].dtype) for i in (0, 1)]
            if self.e4m3:
                both = torch.stack(scales, dim=1)
                scales = [both[:, 0], both[:, 1]]
        self.cache = A.KVCache(*pools, *scales, head_dim=self.d)
        ints = lambda x: cuda(x, torch.int32)
        self.cu_dev, self.kv_dev, self.table_dev = ints(self.cu), ints(np.array(self.kv, dtype=np.int64)), ints(self.table)
        self.batch = A.KVBatch(self.cu_dev, self.kv_dev, self.table_dev, max(self.rows, default=0))
        return self.cache, self.batch


def attend(A, b, q, lse=True, scale=0.0, workspace=None):
    """(o, lse) of the library as device tensors, NaN where nothing was written."""
    import torch
    o = torch.full_like(q, float("nan"), memory_format=torch.contiguous_format)
    l = torch.full((q.shape[1], q.shape[0]), float("nan"), device="cuda") if lse else None
    if workspace is None:
        workspace = torch.full((max(A.attn_paged_workspace_bytes(b.cache, b.batch, q.shape[0], q.shape[1]), 16),), 255, dtype=torch.uint8, device="cuda")
    A.attn_paged_fwd(b.cache, b.batch, q, o, l, workspace, scale)
    return o, l
