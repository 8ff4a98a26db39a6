"""Caches with ragged contexts for the tests of the operators over a long context."""

import numpy as np
import torch

from oracle import cache as oc
from paper_2603_04427_gb300 import binding as tb

FORMATS = {"bf16": {}, "int8": dict(k_int8=True), "int4": dict(k_int4=True)}


class Cache:
    """A cache of random keys and values; the slots past each context hold NaNs (or odd codes), and a
    paged one has pages that nobody owns."""

    def __init__(self, lens, h_q, h_kv, r, d_v, cap, ps=0, k="bf16", seed=0, device="cuda"):
        gen = torch.Generator(device="cpu").manual_seed(seed)
        self.lens, self.r, self.d_v, self.h_q, self.h_kv, self.ps, self.cap = lens, r, d_v, h_q, h_kv, ps, cap
        B = len(lens)
        self.B = B
        table = None
        if ps:
            per = cap // ps
            P = B * per + 3
            table = torch.randperm(P, generator=gen)[:B * per].view(B, per).to(torch.int32)
            kw = dict(page_size=ps, num_pages=P, page_table=table)
        else:
            kw = dict(capacity=cap)
        self.c = tb.ThinKeyCache.allocate(B, h_q, h_kv, r, d_v, device=device, **kw, **FORMATS[k])
        c, self.k = self.c, k
        self.rows_total = c.v.numel() // d_v
        # logical rows: every slot of the caches, then the ones past the context spoilt
        vals = torch.randn(self.rows_total, r, generator=gen)
        code = scale = None
        if k == "bf16":
            flat = vals.to(torch.bfloat16)
        else:
            code, scale = (oc.quantize_int8_per_token if k == "int8" else oc.quantize_int4_per_token)(vals.numpy())
            flat = torch.from_numpy(code if k == "int8" else oc.pack_int4(code))
            scale = torch.from_numpy(scale)
        v = torch.randn(self.rows_total, d_v, generator=gen).to(torch.bfloat16)
        used = torch.zeros(self.rows_total, dtype=torch.bool)
        self.table = None if table is None else table.numpy()
        for b in range(B):
            for g in range(h_kv):
                used[self.rows(b, g)] = True
        v[~used] = float("nan")
        if k == "bf16":
            flat[~used] = float("nan")
        else:
            scale[~used] = float("inf")
            c.k_scale.copy_(scale.view(c.k_scale.shape))
        c.k.copy_(flat.view(c.k.shape))
        c.v.copy_(v.view(c.v.shape))
        self.seq = torch.tensor(lens, dtype=torch.int32, device=device)

    def rows(self, b, g, n=None):
        """Cache rows of the first n tokens (default: the context)."""
        t = np.arange(max(0, min(self.lens[b], self.cap)) if n is None else n)
        if self.ps:
            return (self.table[b][t // self.ps].astype(np.int64) * self.h_kv + g) * self.ps + t % self.ps
        return (b * self.h_kv + g) * self.cap + t

    def keys32(self):
        """Every row's key as the values that the attention sees, float32 [rows, r]."""
        c = self.c
        if self.k == "bf16":
            return c.k.float().cpu().numpy().reshape(-1, self.r)
        code = c.k.cpu().numpy().reshape(self.rows_total, -1)
        code = oc.unpack_int4(code) if self.k == "int4" else code
        with np.errstate(invalid="ignore", over="ignore"):       # spoilt slots
            return code.astype(np.float32) * c.k_scale.cpu().numpy().reshape(-1, 1)

    def keys64(self):
        c = self.c
        if self.k == "bf16":
            return self.keys32().astype(np.float64)
        code = c.k.cpu().numpy().reshape(self.rows_total, -1)
        code = oc.unpack_int4(code) if self.k == "int4" else code
        with np.errstate(invalid="ignore"):
            return code.astype(np.float64) * c.k_scale.cpu().numpy().reshape(-1, 1).astype(np.float64)

    def values(self):
        return self.c.v.float().cpu().numpy().astype(np.float64).reshape(-1, self.d_v)

    def block_rows(self, block):
        """Place of each block's bounds: [b][g] -> array over the context's blocks."""
        return [[self.rows(b, g)[::block] // block for g in range(self.h_kv)] for b in range(self.B)]


def i32(x, device="cuda"):
    return torch.tensor(x, dtype=torch.int32, device=device)


def bits(t):
    """Bit patterns, to compare with NaNs."""
    t = t.detach().cpu().contiguous()
    return t.view({2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()])
