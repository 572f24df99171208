"""Paged caches for the GPU tests: a pool filled with garbage, pages in no order, and what the oracle says that the cache holds."""

from __future__ import annotations

import numpy as np
import torch

import paper_2510_19482_b200 as elutq
from oracle import attention

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def rounded(x: np.ndarray, dtype: str) -> np.ndarray:
    """fp32 values that the 16-bit type holds."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TYPES[dtype]).float().numpy()


def dev(x: np.ndarray, dtype: str) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TYPES[dtype]).cuda()


def ints(x) -> torch.Tensor:
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def garbage(shape, dtype, rng):
    """Bytes of every kind: infinities, NaN, large values."""
    n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    return torch.from_numpy(rng.integers(0, 256, n, dtype=np.uint8)).cuda().view(dtype).reshape(shape)


class Paged:
    """lens: tokens of the sequences; the cache holds k, v (fp32 [tokens, heads, D], lists) as the oracle stores them."""

    def __init__(self, rng, fmt, dtype, lens, heads, D, page, k=None, v=None, factors=True, spare=2):
        self.fmt, self.dtype, self.lens, self.heads, self.D, self.page = fmt, dtype, lens, heads, D, page
        need = [-(-n // page) for n in lens]
        pages = max(1, sum(need) + spare)
        order = rng.permutation(pages)
        wide = max(1, max(need))
        self.table = np.full((len(lens), wide), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at : at + n]
            at += n
        width, kind = {0: (D, TYPES[dtype]), 1: (D, torch.uint8), 2: (D // 2, torch.uint8)}[fmt]
        self.data = [garbage((pages, heads, page, width), kind, rng) for _ in range(2)]
        self.scales = [garbage((pages, heads, page, D // 16), torch.uint8, rng) for _ in range(2)] if fmt == 2 else [None, None]
        self.factors = [rng.uniform(0.3, 3.0, heads).astype(np.float32) if factors and fmt else None for _ in range(2)]
        self.held = []
        for i, x in enumerate((k, v)):
            per = []
            for b, n in enumerate(lens):
                if x is None or n == 0:
                    per.append(np.zeros((n, heads, D)))
                    continue
                if fmt == 0:
                    val = rounded(x[b], dtype)
                    parts = [(self.data[i], dev(x[b], dtype))]
                    per.append(val.astype(np.float64))
                else:
                    codes, scales = attention.stored(x[b], fmt, self.factors[i])
                    parts = [(self.data[i], torch.from_numpy(codes).cuda())] + ([(self.scales[i], torch.from_numpy(scales).cuda())] if fmt == 2 else [])
                    per.append(attention.held(codes, scales, fmt, self.factors[i]))
                slots = torch.from_numpy(self.slots(b, np.arange(n)).astype(np.int64)).cuda()
                for pool, rows in parts:
                    pool[slots // page, :, slots % page] = rows
            self.held.append(per)
        f = [None if x is None else torch.from_numpy(x).cuda() for x in self.factors]
        self.cache = elutq.KvCache(fmt, TYPES[dtype], self.data[0], self.data[1], self.scales[0], self.scales[1], k_factor=f[0], v_factor=f[1])
        self.table_d, self.lens_d = ints(self.table), ints(lens)

    def slots(self, b, pos):
        pos = np.asarray(pos)
        return self.table[b, pos // self.page] * self.page + pos % self.page

    def bytes_at(self, i, slots):
        """What the pool holds at slots: [data] or [codes, scales]."""
        s = torch.from_numpy(np.asarray(slots, dtype=np.int64)).cuda()
        return [p[s // self.page, :, s % self.page].cpu() for p in (self.data[i], self.scales[i]) if p is not None]
