"""Long contexts of one attention layer, decoded in part and kept in part.

    python examples/long_context.py

A decode step of ``SparseServer`` reads a few blocks of each context: tk_block_bounds (of the block
that got the new token), tk_block_select (the blocks whose keys can score highest), tk_attn_decode_blocks.
``BudgetServer`` reads all of a context but keeps it short: tk_attn_weights adds up the attention
that every cached token gets, and now and then tk_cache_evict cuts the contexts to the tokens that
got most and the latest ones; their pages go back to the pool.
The layer's input and weights are random; projections are plain matrix products.
"""

from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2603_04427_gb300 import binding as tk  # noqa: E402
from rope_layer import Layer, Server  # noqa: E402


class _Server(Server):
    """A Server whose tokens are rotated by their own positions: after an eviction the cache holds
    fewer tokens than a sequence has had."""

    def __init__(self, layer, batch, max_len, **kw):
        super().__init__(layer, batch, max_len, **kw)
        self.seen = torch.zeros(batch, dtype=torch.int32, device="cuda")      # tokens a sequence has had
        self.old = torch.zeros(batch, dtype=torch.int32, device="cuda")       # cached before the step
        self.append = tk.prepare_qk_norm_rope_append(
            self.cache, layer.plan, *layer.heads(self.packed), self.seen[:, None], self.slots, self.q,
            q_weight=layer.norm_q, k_weight=layer.norm_k)

    def admit(self, prompts):
        short = (self.seen != self.pool.seq_lens).tolist()
        if any(s and x is not None for s, x in zip(short, prompts)):
            raise RuntimeError("a prompt goes on from its sequence's cached tokens: not after some were evicted")
        self.old.copy_(self.pool.seq_lens)
        outs = super().admit(prompts)
        self.seen += self.pool.seq_lens - self.old
        return outs

    def finish(self, which):
        super().finish(which)
        self.seen[which] = 0

    def decode(self, x):
        torch.matmul(x, self.layer.w, out=self.packed.view(self.batch, -1))
        self.tables()
        self.old.copy_(self.pool.seq_lens)
        self.keep_step()
        self.append()
        self.seen += self.new
        self.attend(self.q.view(self.batch, self.layer.h_q, -1))
        return self.out


class SparseServer(_Server):
    """Decodes over n_select blocks (pages) of each context and kv head: the first, the last, and
    those that can score highest."""

    def __init__(self, layer, batch, max_len, n_select, **kw):
        super().__init__(layer, batch, max_len, **kw)
        self.bounds = tk.block_bounds(self.cache)
        self.pick = tk.BlockSelection.allocate(self.cache, n_select, ids=True)
        self.workspace = tk.decode_blocks_workspace(self.cache, self.pick)

    def admit(self, prompts):
        outs = super().admit(prompts)
        tk.tk_block_bounds(self.cache, self.bounds, self.pool.seq_lens, self.old)
        return outs

    def attend(self, q):
        tk.tk_block_bounds(self.cache, self.bounds, self.pool.seq_lens, self.old, max_new=1)
        tk.tk_block_select(self.cache, q, self.bounds, self.pool.seq_lens, self.max_len, self.pick)
        tk.tk_attn_decode_blocks(self.cache, q, self.pick, self.out, self.workspace)


class BudgetServer(_Server):
    """Keeps at most `keep` tokens of a context, the last `recent` among them, once it has grown to
    keep + slack; window: queries at a prompt's end whose attention is its tokens' first weight."""

    def __init__(self, layer, batch, max_len, keep, recent, slack=16, window=16, **kw):
        super().__init__(layer, batch, max_len, **kw)
        self.keep, self.recent, self.slack, self.window, self.steps = keep, recent, slack, window, 0
        self.weights = tk.slot_weights(self.cache)
        self.weights_ws = tk.attn_weights_workspace(self.cache, max_len)
        self.evict_ws = tk.cache_evict_workspace(self.cache, keep)
        self.kept = torch.empty(batch, layer.h_kv, keep, dtype=torch.int32, device="cuda")

    def admit(self, prompts):
        outs = super().admit(prompts)
        layer = self.layer
        tails = [0 if x is None else min(self.window, x.shape[0]) for x in prompts]
        # a call for the prompts of each number of queries: those of a prompt that goes on from
        # cached tokens are its own alone
        for n in sorted(set(tails) - {0}):
            # the prompts' last queries, again (a real engine has them at hand)
            q = torch.zeros(self.batch, layer.h_q, n, layer.r, dtype=torch.bfloat16, device="cuda")
            for b, x in enumerate(prompts):
                if tails[b] == n:
                    pos = self.seen[b] - n + torch.arange(n, dtype=torch.int32, device="cuda")
                    q[b] = layer.rotated((x[-n:] @ layer.w)[None], pos[None])[0][0]
            # the other sequences keep their weights, or get them by a call of their own
            these = torch.tensor([t == n for t in tails], device="cuda")
            lens = torch.where(these, self.pool.seq_lens, 0).to(torch.int32)
            tk.tk_attn_weights(self.cache, q, lens, self.max_len, self.weights,
                               tk.attn_weights_workspace(self.cache, self.max_len, n), old_lens=self.old)
        self.evict()
        return outs

    def attend(self, q):
        tk.tk_attn_decode(self.cache, q, self.pool.seq_lens, self.max_len, self.out, self.workspace)
        tk.tk_attn_weights(self.cache, q, self.pool.seq_lens, self.max_len, self.weights, self.weights_ws,
                           old_lens=self.old)
        self.steps += 1
        if self.steps % self.slack == 0:
            self.evict()

    def evict(self):
        tk.tk_cache_evict(self.cache, self.pool.seq_lens, self.max_len, self.weights, self.keep, self.recent,
                          self.evict_ws, kept=self.kept, pool=self.pool)


def main():
    layer = Layer()
    d_model = layer.w.shape[0]
    lens, steps, max_len = [700, 33, 250], 48, 1024
    full = Server(layer, len(lens), max_len=max_len)
    sparse = SparseServer(layer, len(lens), max_len, n_select=24)
    budget = BudgetServer(layer, len(lens), max_len, keep=256, recent=32)
    tokens = [torch.randn(n + steps, d_model, device="cuda").to(torch.bfloat16) for n in lens]
    for s in (full, sparse, budget):
        s.admit([t[:n] for t, n in zip(tokens, lens)])
    off = {"blocks": 0.0, "budget": 0.0}
    for i in range(steps):
        x = torch.stack([t[n + i] for t, n in zip(tokens, lens)])
        ref = full.decode(x)
        for name, s in (("blocks", sparse), ("budget", budget)):
            off[name] = max(off[name], float((s.decode(x) - ref).norm() / ref.norm()))
    if tk.tk_get_device_error() != 0:
        raise RuntimeError("device error word set")
    print(f"decoded {steps} tokens of contexts {lens}: over 24 blocks of 16 tokens off by {off['blocks']:.2f} of the "
          f"output, with {budget.keep} tokens kept by {off['budget']:.2f} (random weights: attention is nearly flat)")
    print(f"cached tokens {full.pool.seq_lens.tolist()} and {budget.pool.seq_lens.tolist()}, "
          f"free pages {full.pool.free_count.item()} and {budget.pool.free_count.item()}")
    return off


if __name__ == "__main__":
    from paper_2603_04427_gb300 import build
    build.build()
    main()
