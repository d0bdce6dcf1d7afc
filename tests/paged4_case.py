"""Random problems over a paged cache in 4 bits, as paged_case has them for the other types."""

import numpy as np
import torch

import oracle.paged as ref
from paged_case import Case, h64
from paper_2606_10537_amd._lib import PD_FP4_E2M1


def pack4(codes):
    """Codes [..., d] as bytes [..., d / 2]."""
    codes = np.asarray(codes)
    return torch.from_numpy((codes[..., ::2] + 16 * codes[..., 1::2]).astype(np.uint8))


def unpack4(x):
    x = np.asarray(x)
    return np.stack([x & 15, x >> 4], -1).reshape(*x.shape[:-1], 2 * x.shape[-1])


class Case4(Case):
    """A Case whose pages hold E2M1 values: everything that no sequence holds is 0x77, its exponent bytes 255 (NaN)."""

    def __init__(self, lens, **kw):
        super().__init__(lens, cache=PD_FP4_E2M1, **kw)

    def place(self):
        d = self.dims
        super().place()                                     # the bounds
        pool = (d.n_pages, d.n_heads_kv, d.page_rows, d.head_dim // 2)
        self.held = {"k": [], "v": []}
        for n, rows in (("k", self.k_rows), ("v", self.v_rows)):
            p = torch.full(pool, 0x77, dtype=torch.uint8)
            e = torch.full((d.n_pages, d.n_heads_kv, d.head_dim // 32, d.page_rows), 255, dtype=torch.uint8)
            for b, x in enumerate(rows):
                codes, ex = ref.quantise4_ref(h64(x))
                self.held[n].append(ref.held4_ref(codes, ex))
                byte = pack4(codes)
                for r in range(len(x)):
                    pg, sl = int(self.table[b, r // d.page_rows]), r % d.page_rows
                    p[pg, :, sl] = byte[r]
                    e[pg, :, :, sl] = torch.from_numpy(ex[r] + 127).to(torch.uint8)
            self.pool[n], self.pool[n + "_exp"] = p, e
