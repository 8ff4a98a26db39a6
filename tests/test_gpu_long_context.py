"""The operators over a long context together, as a server calls them (examples/long_context.py)."""

import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from _helpers import f64, parity, require_gpu
from oracle import attention as oa
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    require_gpu()
    spec = importlib.util.spec_from_file_location("long_context", os.path.join(ROOT, "examples", "long_context.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    tb.tk_get_device_error()
    yield m
    assert tb.tk_get_device_error() == 0


def _tokens(lens, steps, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n + steps, d, device="cuda", generator=g).to(torch.bfloat16) for n in lens]


def _layer(ex, **kw):
    return ex.Layer(d_model=128, **dict(dict(h_q=8, h_kv=2, r=32, d_v=64, seed=3), **kw))


@pytest.mark.parametrize("k_int8", [False, True])
def test_all_blocks_chosen_is_the_whole_context(ex, k_int8):
    """With room for every block the sparse step is the full one, token after token, across block
    boundaries, with a sequence that starts empty and one that ends."""
    layer, lens, steps = _layer(ex), [1, 100, 33], 40
    full = ex.Server(layer, 3, max_len=160, k_int8=k_int8)
    part = ex.SparseServer(layer, 3, 160, n_select=10, k_int8=k_int8)
    tokens = _tokens(lens, steps, 128, 1)
    for s in (full, part):
        s.admit([t[:n] for t, n in zip(tokens, lens)])
    for i in range(steps):
        if i == 20:
            for s in (full, part):
                s.finish([1])
        x = torch.stack([t[n + i] for t, n in zip(tokens, lens)])
        a, b = full.decode(x), part.decode(x)
        parity(f64(b), f64(a))
    assert part.pool.seq_lens.tolist() == [41, 0, 73]


def test_chosen_blocks_hold_the_largest_scores(ex):
    """Each step's choice: no block left out has a key that scores above the bound of every chosen
    one, and the output is the attention over the chosen tokens."""
    layer = _layer(ex)
    s = ex.SparseServer(layer, 2, 512, n_select=6)
    tokens = _tokens([400, 123], 5, 128, 2)
    s.admit([t[:n] for t, n in zip(tokens, [400, 123])])
    for i in range(5):
        out = s.decode(torch.stack([t[n + i] for t, n in zip(tokens, [400, 123])]))
        q, keys, vals = f64(s.q)[:, :, 0], f64(s.cache.k), f64(s.cache.v)
        for b, L in enumerate((400 + i + 1, 123 + i + 1)):
            pages = s.pool.page_table[b, :-(-L // 16)].tolist()
            for g in range(2):
                k = np.concatenate([keys[p, g] for p in pages])[:L]
                v = np.concatenate([vals[p, g] for p in pages])[:L]
                ids = s.pick.ids[b, g].tolist()
                assert ids[0] == 0 and ids[-1] == len(pages) - 1 and ids == sorted(set(ids)) and len(ids) == 6
                t = np.concatenate([np.arange(16 * j, min(16 * j + 16, L)) for j in ids])
                ref = oa.attention_head(q[b, 4 * g:4 * g + 4], k[t], v[t], 1 / math.sqrt(32))
                parity(f64(out)[b, 4 * g:4 * g + 4], ref)


def test_a_budget_that_is_never_reached_changes_nothing(ex):
    layer, lens = _layer(ex), [50, 7]
    full, part = ex.Server(layer, 2, max_len=160), ex.BudgetServer(layer, 2, 160, keep=150, recent=8, slack=4)
    tokens = _tokens(lens, 20, 128, 3)
    for s in (full, part):
        s.admit([t[:n] for t, n in zip(tokens, lens)])
    for i in range(20):
        x = torch.stack([t[n + i] for t, n in zip(tokens, lens)])
        assert torch.equal(full.decode(x), part.decode(x))
    assert full.pool.seq_lens.tolist() == part.pool.seq_lens.tolist()
    assert full.pool.free_count.item() == part.pool.free_count.item()
    # every query adds a weight of one for each of the kv head's four query heads
    total = torch.zeros(2, 2, dtype=torch.float64)
    for b, n in enumerate(lens):
        for p, page in enumerate(part.pool.page_table[b, :-(-(n + 20) // 16)].tolist()):
            total[b] += part.weights[page, :, :min(16, n + 20 - 16 * p)].double().sum(-1).cpu()
    want = torch.tensor([[4.0 * (16 + 20)] * 2, [4.0 * (7 + 20)] * 2], dtype=torch.float64)
    # sums of at most 36 positive terms a token in 32 bits, each weight within 1e-5 (test_gpu_attn_weights.py)
    assert torch.allclose(total, want, rtol=2e-5)


@pytest.mark.parametrize("k_int8", [False, True])
def test_budget_server_against_a_list_of_kept_tokens(ex, k_int8):
    """Follows each kv head's tokens through prompts, steps and evictions by `kept`: the cache holds
    what those tokens were cached as, the output is the attention over them, the pool its pages."""
    layer, lens, keep, recent, slack, steps = _layer(ex, r=32), [150, 9, 60], 64, 10, 6, 30
    s = ex.BudgetServer(layer, 3, 192, keep=keep, recent=recent, slack=slack, k_int8=k_int8)
    full = ex.Server(layer, 3, max_len=192, k_int8=k_int8)      # all tokens, for what each was cached as
    tokens = _tokens(lens, steps, 128, 4)
    mine = [[list(range(n)) for _ in range(2)] for n in lens]

    def after_eviction():
        kept = s.kept.cpu().numpy()
        for b in range(3):
            for g in range(2):
                if len(mine[b][g]) > keep:
                    mine[b][g] = [mine[b][g][j] for j in kept[b, g]]
                    n = int(s.seen[b])
                    assert mine[b][g][-recent:] == list(range(n - recent, n))

    def rows(server, b, n):
        return server.pool.page_table[b, :-(-n // 16)].tolist()

    for x in (s, full):
        x.admit([t[:n] for t, n in zip(tokens, lens)])
    after_eviction()
    for i in range(steps):
        x = torch.stack([t[n + i] for t, n in zip(tokens, lens)])
        full.decode(x)
        for b in range(3):
            for g in range(2):
                mine[b][g].append(lens[b] + i)
        attended = [[list(m) for m in mine[b]] for b in range(3)]
        out = s.decode(x)
        code = lambda c: c.k.float() * c.k_scale[..., None] if k_int8 else c.k.float()  # noqa: E731
        all_k, all_v = code(full.cache).cpu().double().numpy(), f64(full.cache.v)
        q = f64(s.q)[:, :, 0]
        for b in range(3):
            n = lens[b] + i + 1
            for g in range(2):
                k = np.concatenate([all_k[p, g] for p in rows(full, b, n)])[attended[b][g]]
                v = np.concatenate([all_v[p, g] for p in rows(full, b, n)])[attended[b][g]]
                parity(f64(out)[b, 4 * g:4 * g + 4], oa.attention_head(q[b, 4 * g:4 * g + 4], k, v, 1 / math.sqrt(32)))
        if (i + 1) % slack == 0:
            after_eviction()
        k_now, v_now = code(s.cache).cpu().double().numpy(), f64(s.cache.v)
        held = 0
        for b in range(3):
            n = lens[b] + i + 1
            assert s.pool.seq_lens[b].item() == len(mine[b][0]) == len(mine[b][1])
            pages = rows(s, b, len(mine[b][0]))
            held += len(pages)
            for g in range(2):
                for now, was in ((k_now, all_k), (v_now, all_v)):
                    a = np.concatenate([now[p, g] for p in pages])[:len(mine[b][g])]
                    assert np.array_equal(a, np.concatenate([was[p, g] for p in rows(full, b, n)])[mine[b][g]])
        assert s.pool.free_count.item() == s.cache.desc.num_pages - held


def test_a_further_prompt_after_an_eviction_is_refused(ex):
    s = ex.BudgetServer(_layer(ex), 1, 192, keep=64, recent=10)
    s.admit([_tokens([100], 0, 128, 5)[0]])
    assert s.pool.seq_lens.tolist() == [64]
    with pytest.raises(RuntimeError):
        s.admit([_tokens([10], 0, 128, 6)[0]])
    s.finish([0])
    s.admit([_tokens([20], 0, 128, 7)[0]])
    assert s.pool.seq_lens.tolist() == [20] == s.seen.tolist()


def test_example_runs(ex):
    off = ex.main()
    assert set(off) == {"blocks", "budget"} and all(math.isfinite(v) for v in off.values())
