"""One attention layer with per-head norm and rotation, served and trained.

    python examples/rope_layer.py

Serving: ragged prompts are admitted to a paged cache and decoded token by token.  A step is
tk_block_tables (pages, slots, positions), then for a prompt tk_qk_norm_rope and
tk_attn_prefill_cached, for single tokens tk_qk_norm_rope_append and tk_attn_decode.
Training: tk_qk_norm_rope, tk_attn_forward, tk_attn_backward, tk_qk_norm_rope_backward.
The layer's input and weights are random; projections are plain matrix products.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2603_04427_gb300 import binding as tk  # noqa: E402

BF16 = torch.bfloat16


class Layer:
    """Thin keys (r wide), grouped queries, one packed projection, norm weights of q and k."""

    def __init__(self, d_model=512, h_q=16, h_kv=4, r=32, d_v=64, seed=0):
        self.h_q, self.h_kv, self.r, self.d_v = h_q, h_kv, r, d_v
        self.widths = [h_q * r, h_kv * r, h_kv * d_v]
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w = (torch.randn(d_model, sum(self.widths), device="cuda", generator=g) / d_model ** 0.5).to(BF16)
        self.norm_q = 1 + 0.1 * torch.randn(r, device="cuda", generator=g)
        self.norm_k = 1 + 0.1 * torch.randn(r, device="cuda", generator=g)
        self.plan = tk.rope_plan(r)

    def heads(self, packed):
        """q, k, v [B, H, S, width] as views of packed rows [B, S, all heads]."""
        B, S, _ = packed.shape
        parts = packed.split(self.widths, dim=-1)
        return [t.view(B, S, h, -1).transpose(1, 2) for t, h in zip(parts, (self.h_q, self.h_kv, self.h_kv))]

    def rotated(self, packed, positions):
        """q, k, v as the attention's prefill reads them: normalised, rotated, head-major."""
        q, k, v = self.heads(packed)
        out = [torch.empty(t.shape, dtype=BF16, device="cuda") for t in (q, k, v)]
        tk.tk_qk_norm_rope(self.plan, q, k, v, positions, *out, q_weight=self.norm_q, k_weight=self.norm_k)
        return out


class Server:
    """A paged cache of the layer, its page pool, and the buffers of a decode step."""

    def __init__(self, layer, batch, max_len=512, page_size=16, num_pages=None, k_int8=False):
        self.layer, self.batch, self.max_len = layer, batch, max_len
        max_pages = -(-max_len // page_size)
        num_pages = num_pages or batch * max_pages
        self.pool = tk.PagePool.allocate(batch, max_pages, page_size, num_pages)
        self.cache = tk.ThinKeyCache.allocate(batch, layer.h_q, layer.h_kv, layer.r, layer.d_v, page_size=page_size,
                                              num_pages=num_pages, page_table=self.pool.page_table, k_int8=k_int8)
        i32 = dict(dtype=torch.int32, device="cuda")
        # a decode step's fixed buffers, its two prepared calls, and the attention's workspace
        self.new = torch.zeros(batch, **i32)      # 1 for the sequences that are being served
        self.slots, self.pos = torch.empty(batch, **i32), torch.empty(batch, **i32)
        self.packed = torch.empty(batch, 1, sum(layer.widths), dtype=BF16, device="cuda")
        self.q = torch.empty(batch, layer.h_q, 1, layer.r, dtype=BF16, device="cuda")
        self.out = torch.empty(batch, layer.h_q, layer.d_v, device="cuda")
        self.workspace = tk.decode_workspace(self.cache.desc, max_len)
        # lengths and free pages after a step, the pool's own only once nothing was refused
        self.lens, self.free, self.refused = torch.empty(batch, **i32), torch.empty(1, **i32), torch.empty(1, **i32)
        self.after = dict(seq_lens_out=self.lens, free_count_out=self.free, refused=self.refused)
        self.tables = tk.prepare_block_tables(self.pool, self.new, self.slots, self.pos, tokens_per_seq=1, **self.after)
        self.append = tk.prepare_qk_norm_rope_append(
            self.cache, layer.plan, *layer.heads(self.packed), self.pos[:, None], self.slots, self.q,
            q_weight=layer.norm_q, k_weight=layer.norm_k)

    def keep_step(self):
        """Takes over the step that tk_block_tables worked out, or, if a request was refused, leaves it: a step in
        which nobody finishes writes only what the old lengths and free count leave unused."""
        if self.refused.item():
            raise RuntimeError("the page pool, or a row of the page table, does not hold this step")
        self.pool.seq_lens.copy_(self.lens)
        self.pool.free_count.copy_(self.free)

    def admit(self, prompts):
        """Prompts, one [tokens, d_model] per sequence (None: idle) -> attention outputs, head-major.  Raises, and
        changes nothing, if one of them does not fit."""
        lens = [0 if x is None else x.shape[0] for x in prompts]
        i32 = dict(dtype=torch.int32, device="cuda")
        before = self.pool.seq_lens.clone()
        slots, pos = torch.empty(sum(lens), **i32), torch.empty(sum(lens), **i32)
        tk.tk_block_tables(self.pool, torch.tensor(lens, **i32), slots, pos, **self.after)
        self.keep_step()
        layer, outs, row = self.layer, [], 0
        for b, x in enumerate(prompts):
            if x is None:
                outs.append(None)
                continue
            n = lens[b]
            q, k, v = layer.rotated((x @ layer.w)[None], pos[row:row + n][None])
            d = self.cache.desc
            one = tk.ThinKeyCache(
                tk.tk_cache_desc(1, d.h_q, d.h_kv, d.r, d.d_v, 0, d.page_size, d.num_pages, d.max_pages_per_seq,
                                 d.k_dtype),
                self.cache.k, self.cache.v, self.cache.k_scale, self.pool.page_table[b:b + 1])
            out = torch.empty(1, layer.h_q, n, layer.d_v, device="cuda")
            tk.tk_attn_prefill_cached(one, q, k, v, before[b:b + 1], self.max_len, out)
            outs.append(out)
            row += n
            self.new[b] = 1
        return outs

    def decode(self, x):
        """One token per served sequence, x [batch, d_model] -> attention output [batch, h_q, d_v], zero for the
        others.  Raises, and changes nothing, if one of them does not fit."""
        torch.matmul(x, self.layer.w, out=self.packed.view(self.batch, -1))
        self.tables()
        self.keep_step()
        self.append()
        return tk.tk_attn_decode(self.cache, self.q.view(self.batch, self.layer.h_q, -1), self.pool.seq_lens,
                                 self.max_len, self.out, self.workspace)

    def finish(self, which):
        """Gives back the pages of the sequences in `which`, which then stay empty until prompts are admitted."""
        self.new[which] = 0
        new = torch.zeros(self.batch, dtype=torch.int32, device="cuda")
        new[which] = -1
        empty = torch.empty(0, dtype=torch.int32, device="cuda")
        tk.tk_block_tables(self.pool, new, empty, empty)


def train_step(layer, x, d_out):
    """Gradients of the packed projection's output and of the norm weights for dL/d(attention output)."""
    B, S, _ = x.shape
    packed = x @ layer.w
    positions = torch.arange(S, dtype=torch.int32, device="cuda").expand(B, S)
    q, k, v = layer.rotated(packed, positions)
    out = torch.empty(B, layer.h_q, S, layer.d_v, dtype=BF16, device="cuda")
    lse = torch.empty(B, layer.h_q, S, device="cuda")
    tk.tk_attn_forward(q, k, v, out, lse)
    grads = [torch.empty(t.shape, device="cuda") for t in (q, k, v)]
    tk.tk_attn_backward(q, k, v, out, d_out, lse, *grads)
    d_packed = torch.empty_like(packed)
    d_norm_q, d_norm_k = torch.empty_like(layer.norm_q), torch.empty_like(layer.norm_k)
    raw_q, raw_k, _ = layer.heads(packed)
    tk.tk_qk_norm_rope_backward(layer.plan, raw_q, raw_k, positions, *grads, *layer.heads(d_packed),
                                q_weight=layer.norm_q, k_weight=layer.norm_k, dq_weight=d_norm_q,
                                dk_weight=d_norm_k)
    return out, d_packed, d_norm_q, d_norm_k


def main():
    layer = Layer()
    d_model = layer.w.shape[0]
    lens, steps = [37, 1, 130], 20
    server = Server(layer, len(lens))
    tokens = [torch.randn(n + steps, d_model, device="cuda").to(BF16) for n in lens]
    server.admit([t[:n] for t, n in zip(tokens, lens)])
    last = None
    for i in range(steps):
        last = server.decode(torch.stack([t[n + i] for t, n in zip(tokens, lens)]))
    # the same tokens in one causal prefill: its last row is the last decode step
    worst = 0.0
    for b, t in enumerate(tokens):
        pos = torch.arange(t.shape[0], dtype=torch.int32, device="cuda")[None]
        q, k, v = layer.rotated((t @ layer.w)[None], pos)
        out = torch.empty(1, layer.h_q, t.shape[0], layer.d_v, device="cuda")
        tk.tk_attn_prefill(q, k, v, out)
        worst = max(worst, float((out[0, :, -1] - last[b]).abs().max()))
    server.finish([0, 2])
    print(f"served {sum(lens)} prompt and {steps * len(lens)} decoded tokens; "
          f"largest difference from one prefill {worst:.1e}; "
          f"lengths {server.pool.seq_lens.tolist()}, free pages {server.pool.free_count.item()}")
    x = torch.randn(2, 256, d_model, device="cuda").to(BF16)
    out, d_packed, d_norm_q, _ = train_step(layer, x, torch.randn(2, layer.h_q, 256, layer.d_v, device="cuda").to(BF16))
    print(f"trained: |d packed| {float(d_packed.float().norm()):.3f}, |d norm_q| {float(d_norm_q.norm()):.3f}")
    if tk.tk_get_device_error() != 0:
        raise RuntimeError("device error word set")
    return worst


if __name__ == "__main__":
    from paper_2603_04427_gb300 import build
    build.build()
    main()
