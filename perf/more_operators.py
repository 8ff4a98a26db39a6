"""What is measured of the operators that let a decode step read, and a cache keep, only a part of a
long context: bounds of key blocks, the choice of blocks for each query, the decode over the chosen
blocks, accumulated attention weights, and eviction by them.

A case's ``op`` says which operator it is a pass of:

``bounds``   element-wise minimum and maximum of the keys of every block that got new tokens.
``select``   per sequence and kv head: the blocks whose keys can score highest with the step's queries.
``decode``   one decode step over the chosen blocks alone.
``weights``  the attention weights of a step's queries, added up per cached token.
``evict``    the tokens of a longer context that stay, moved to the front of the cache.
"""

import math

import torch

own = False


# ------------------------------------------------------------------------------------- cases

def _case(name, op, batch, h_q, h_kv, r, ctx, **kw):
    c = dict(name=name, op=op, batch=batch, h_q=h_q, h_kv=h_kv, r=r, ctx=ctx, d_v=128, k="bf16", page=0)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of 16 sequences of the Mistral shape: the block of each new token; latency
        _case("bounds_decode_b16", "bounds", 16, 32, 8, 32, 4096, block=64, new=1),
        # one long document with full-width keys, once after its prefill
        _case("bounds_document_131071", "bounds", 1, 8, 8, 128, 131071, block=64, new=131071),
        # a decode step of 16 sequences: 32 of up to 512 blocks; latency
        _case("select_b16_ctx32k", "select", 16, 32, 8, 32, 32768, block=64, n_select=32),
        # few long contexts in small pages: up to 8192 blocks for each kv head
        _case("select_b4_ctx128k_page16", "select", 4, 32, 8, 32, 131072, block=16, page=16, n_select=128),
        # many sequences of a multi-head model with wider keys, a quarter of the context read
        _case("select_b37_mha_ctx64k", "select", 37, 16, 16, 64, 65536, block=64, n_select=256),
        # a decode step of 16 sequences that reads 64 blocks of 64 tokens of each kv head
        _case("decode_b16_64_blocks", "decode", 16, 32, 8, 32, 32768, block=64, n_select=64),
        # odd batch, int8 keys, pages of 32 tokens, one query head per kv head, narrow values
        _case("decode_int8_b7_page32", "decode", 7, 4, 4, 64, 16384, block=32, page=32, n_select=100, k="int8", d_v=64),
        # a decode step's weights on every cached token of 16 sequences
        _case("weights_decode_b16", "weights", 16, 32, 8, 32, 4096, queries=1, decay=1.0),
        # the same of four very long contexts in pages, the largest; older steps fade
        _case("weights_decode_b4_ctx128k", "weights", 4, 32, 8, 32, 131072, page=64, queries=1, decay=0.99),
        # the last 32 queries of two prompts say which of its tokens matter
        _case("weights_window_32", "weights", 2, 32, 8, 64, 16381, queries=32, decay=0.0),
        # now and then in a decode with a budget of 4096 tokens: 256 go, the last 128 always stay
        _case("evict_decode_b16", "evict", 16, 32, 8, 32, 4352, keep=4096, recent=128),
        # three prompts cut to an eighth, int8 keys of full width, paged
        _case("evict_prompt_int8_b3", "evict", 3, 16, 4, 128, 32761, keep=4095, recent=33, k="int8", page=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["bounds", "select", "select", "decode", "weights", "weights", "evict", "evict"])
    r = rng.choice([16, 32, 64, 128])
    h_kv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, h_kv=h_kv, h_q=h_kv * rng.choice([1, 2, 4, 8]), r=r, d_v=rng.choice([64, 128]),
             k=rng.choice(["bf16", "bf16", "int8", "int4"] if r >= 32 else ["bf16", "int8"]))
    c["batch"] = _log_int(rng, 1, 48)
    # cached keys of the whole batch stay below those of the largest listed case
    top = min(65536, (1 << 27) // (c["batch"] * h_kv * r))
    c["ctx"] = _log_int(rng, 64, max(65, top))
    c["page"] = rng.choice([0, 0, 16, 64, 256])
    if op in ("bounds", "select", "decode"):
        c["block"] = c["page"] or rng.choice([16, 32, 64, 128, 256])
        blocks = -(-c["ctx"] // c["block"])
        if op == "bounds":
            c["new"] = rng.choice([1, 1, _log_int(rng, 2, c["ctx"])])
        else:
            c["n_select"] = _log_int(rng, 2, max(3, min(blocks, 512)))
    elif op == "weights":
        c["queries"] = rng.choice([1, 1, 1, 3, 16, 64])
        c["decay"] = rng.choice([0.0, 0.9, 1.0])
    else:
        c["keep"] = _log_int(rng, 32, c["ctx"])
        c["recent"] = rng.choice([0, 1, c["keep"] // 8, c["keep"] // 2])
    return c


# ------------------------------------------------------------------------------------ inputs

def _capacity(case):
    """Token slots of a sequence: whole blocks, or pages."""
    unit = case["page"] or case.get("block", 16)
    return -(-case["ctx"] // unit) * unit


def _make_cache(case, gen, s):
    B, hkv, r, dv, ps = (case[x] for x in ("batch", "h_kv", "r", "d_v", "page"))
    cap = _capacity(case)
    if ps:
        pages = B * (cap // ps)
        lead = (pages, hkv, ps)
        s["table"] = torch.randperm(pages, device="cuda", generator=gen).view(B, -1).to(torch.int32)
    else:
        lead = (B, hkv, cap)
        s["table"] = None
    s["v"] = s["scale_k"] = None
    if case["op"] in ("bounds", "weights", "evict", "decode"):
        if case["k"] == "bf16":
            s["k"] = torch.randn(*lead, r, device="cuda", generator=gen, dtype=torch.bfloat16)
        else:
            if case["k"] == "int8":
                s["k"] = torch.randint(-127, 128, (*lead, r), device="cuda", generator=gen, dtype=torch.int8)
            else:        # two codes of -7 .. 7 a byte
                two = torch.randint(-7, 8, (2, *lead, r // 2), device="cuda", generator=gen, dtype=torch.int8)
                s["k"] = ((two[0] & 15) | (two[1] << 4)).view(torch.uint8)
            peak = 2.0 + torch.rand(lead, device="cuda", generator=gen)
            s["scale_k"] = peak / (127 if case["k"] == "int8" else 7)
    if case["op"] in ("evict", "decode"):
        s["v"] = torch.randn(*lead, dv, device="cuda", generator=gen, dtype=torch.bfloat16)
    s["lead"] = lead


def _own_cache(case, s):
    from paper_2603_04427_gb300 import binding as tk
    ps = case["page"]
    fmt = {"bf16": tk.TK_BF16, "int8": tk.TK_I8, "int4": tk.TK_I4}[case["k"]]
    desc = tk.tk_cache_desc(case["batch"], case["h_q"], case["h_kv"], case["r"], case["d_v"],
                            0 if ps else _capacity(case), ps, s["lead"][0] if ps else 0,
                            s["table"].shape[1] if ps else 0, fmt)
    return tk, tk.ThinKeyCache(desc, s.get("k"), s["v"], s["scale_k"], s["table"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, hq, hkv, r, dv, ctx, op = (case[x] for x in ("batch", "h_q", "h_kv", "r", "d_v", "ctx", "op"))
    s = dict(case=case)
    _make_cache(case, gen, s)
    # ragged contexts, the first of the full length
    lens = torch.randint(ctx - ctx // 4, ctx + 1, (B,), device="cuda", generator=gen)
    lens[0] = ctx
    s["lens"] = lens.to(torch.int32)
    i32 = dict(device="cuda", dtype=torch.int32)
    if op == "bounds":
        new = torch.minimum(lens, torch.full_like(lens, case["new"]))
        s["old"] = (lens - new).to(torch.int32)
        lead = (*s["lead"][:2],) if case["page"] else (B, hkv, _capacity(case) // case["block"])
        s["bounds"] = torch.zeros(*lead, 2, r, device="cuda", dtype=torch.bfloat16)
        if own:
            tk, s["cache"] = _own_cache(case, s)
            s["call"] = tk.prepare_block_bounds(s["cache"], s["bounds"], s["lens"], old_lens=s["old"],
                                                max_new=case["new"], block=case["block"])
    elif op == "select":
        # bounds as neighbouring keys leave them: a centre and a spread for each element of a block
        lead = (*s["lead"][:2],) if case["page"] else (B, hkv, _capacity(case) // case["block"])
        mid = 0.8 * torch.randn(*lead, r, device="cuda", generator=gen)
        half = 0.8 + 1.2 * torch.rand(*lead, r, device="cuda", generator=gen)
        s["bounds"] = torch.stack([mid - half, mid + half], -2).to(torch.bfloat16)
        s["q"] = torch.randn(B, hq, r, device="cuda", generator=gen, dtype=torch.bfloat16)
        n = case["n_select"]
        s["out"] = dict(table=torch.empty(B * hkv, n, **i32), lens=torch.empty(B * hkv, **i32),
                        ids=torch.empty(B, hkv, n, **i32))
        if own:
            tk, s["cache"] = _own_cache(case, s)
            pick = tk.BlockSelection(case["block"], **s["out"])
            s["call"] = tk.prepare_block_select(s["cache"], s["q"], s["bounds"], s["lens"], ctx, pick)
    elif op == "decode":
        # each kv head's chosen blocks in order, the last block of the context among them
        n, bs = case["n_select"], case["block"]
        most = _capacity(case) // bs
        count = (lens + bs - 1) // bs
        key = torch.rand(B, hkv, most, device="cuda", generator=gen)
        j = torch.arange(most, device="cuda")
        key = key.masked_fill((j >= count[:, None])[:, None], -1.0).masked_fill((j == count[:, None] - 1)[:, None], 2.0)
        ids = key.argsort(-1, descending=True)[..., :n]
        took = torch.minimum(count, torch.full_like(count, n))
        ids = torch.where(torch.arange(ids.shape[-1], device="cuda") < took[:, None, None], ids, most).sort(-1).values
        g = torch.arange(hkv, device="cuda")[:, None]
        if case["page"]:
            phys = s["table"].long()[torch.arange(B, device="cuda")[:, None, None], ids.clamp(max=most - 1)] * hkv + g
        else:
            phys = (torch.arange(B, device="cuda")[:, None, None] * hkv + g) * most + ids
        table = torch.full((B, hkv, n), -1, **i32)
        table[..., :ids.shape[-1]] = torch.where(ids < most, phys, -1).to(torch.int32)
        s["pick"] = table.view(B * hkv, n)
        tail = lens - (count - 1) * bs
        s["pick_lens"] = ((took - 1) * bs + tail)[:, None].expand(B, hkv).reshape(-1).to(torch.int32).contiguous()
        s["q"] = (1.5 * torch.randn(B, hq, r, device="cuda", generator=gen)).to(torch.bfloat16)
        s["out"] = torch.empty(B, hq, dv, device="cuda", dtype=torch.bfloat16)
        if own:
            tk, s["cache"] = _own_cache(case, s)
            pick = tk.BlockSelection(bs, s["pick"], s["pick_lens"])
            s["call"] = tk.prepare_attn_decode_blocks(s["cache"], s["q"], pick, s["out"],
                                                      tk.decode_blocks_workspace(s["cache"], pick))
    elif op == "weights":
        n = case["queries"]
        s["q"] = (1.5 * torch.randn(B, hq, n, r, device="cuda", generator=gen)).to(torch.bfloat16)
        s["w"] = torch.rand(s["lead"], device="cuda", generator=gen)
        s["old"] = (lens - n).clamp(min=0).to(torch.int32)
        if own:
            tk, s["cache"] = _own_cache(case, s)
            ws = tk.attn_weights_workspace(s["cache"], ctx, n)
            s["call"] = tk.prepare_attn_weights(s["cache"], s["q"], s["lens"], ctx, s["w"], ws, old_lens=s["old"],
                                                decay=case["decay"])
    else:
        # a few tokens hold most of the attention
        s["w"] = torch.exp(2.0 * torch.randn(s["lead"], device="cuda", generator=gen))
        s["w_out"] = torch.zeros_like(s["w"])
        s["lens_out"] = torch.empty(B, **i32)
        s["kept"] = torch.empty(B, hkv, case["keep"], **i32)
        if own:
            tk, s["cache"] = _own_cache(case, s)
            ws = tk.cache_evict_workspace(s["cache"], case["keep"])
            s["call"] = tk.prepare_cache_evict(s["cache"], s["lens"], ctx, s["w"], case["keep"], case["recent"], ws,
                                               weights_out=s["w_out"], seq_lens_out=s["lens_out"], kept=s["kept"])
    return s


# ------------------------------------------------------------------------------------- plain

def _rows(s, case, tokens):
    """Cache row of each token of tokens [B, 1 or H_kv, n] (any beyond the context: a row that is there)."""
    B, hkv, ps = case["batch"], case["h_kv"], case["page"]
    b = torch.arange(B, device="cuda")[:, None, None]
    g = torch.arange(hkv, device="cuda")[:, None]
    t = tokens.clamp(0, _capacity(case) - 1)
    if ps:
        return (s["table"].long()[b, t // ps] * hkv + g) * ps + t % ps
    return (b * hkv + g) * _capacity(case) + t


def _codes(k):
    """int4 codes, two a byte, as numbers."""
    k = k.to(torch.int32)
    return torch.stack([((k & 15) ^ 8) - 8, ((k >> 4) ^ 8) - 8], -1).flatten(-2)


def _keys(s, case, rows, dtype=torch.float32):
    k = s["k"].view(-1, s["k"].shape[-1])[rows]
    if case["k"] == "bf16":
        return k.to(dtype)
    code = _codes(k) if case["k"] == "int4" else k
    return code.to(dtype) * s["scale_k"].view(-1)[rows].to(dtype)[..., None]


def _outward(x, up):
    """float32 to the bf16 number next to it, upwards or downwards."""
    bits = x.view(torch.int32)
    away = (bits >= 0) if up else (bits < 0)       # growing magnitude is outward
    return (torch.where(away, bits + 0xffff, bits) & -65536).view(torch.float32).to(torch.bfloat16)


def _plain_bounds(s, case):
    bs, hkv = case["block"], case["h_kv"]
    old, lens = s["old"].long(), s["lens"].long()
    n = min((case["new"] - 1) // bs + 2, _capacity(case) // bs)
    blk = (old // bs)[:, None] + torch.arange(n, device="cuda")                 # [B, n]
    at = (blk[..., None] * bs + torch.arange(bs, device="cuda")).flatten(1)     # tokens
    k = _keys(s, case, _rows(s, case, at[:, None])).unflatten(2, (n, bs))       # [B, H, n, bs, r]
    there = (at < lens[:, None])[:, None].unflatten(2, (n, bs))[..., None]
    lo = torch.where(there, k, math.inf).amin(3)
    hi = torch.where(there, k, -math.inf).amax(3)
    both = torch.stack([_outward(lo, False), _outward(hi, True)], -2)           # [B, H, n, 2, r]
    row = _rows(s, case, blk[:, None] * bs) // bs
    live = (blk * bs < lens[:, None])[:, None].expand(-1, hkv, -1)
    s["bounds"].view(-1, 2, case["r"])[row[live]] = both[live]
    return s["bounds"]


def _plain_select(s, case):
    B, hkv, r, bs, n = (case[x] for x in ("batch", "h_kv", "r", "block", "n_select"))
    lens = s["lens"].long()
    most = _capacity(case) // bs
    blk = torch.arange(most, device="cuda")
    row = _rows(s, case, (blk * bs).expand(B, 1, most)) // bs                   # [B, H, most]
    box = s["bounds"].view(-1, 2, r)[row].double()      # scores next to the border: 64 bits
    q = s["q"].view(B, hkv, -1, r).double()
    score = q.clamp(min=0) @ box[..., 1, :].transpose(-1, -2) + q.clamp(max=0) @ box[..., 0, :].transpose(-1, -2)
    score = score.amax(2)
    count = ((lens + bs - 1) // bs)[:, None, None]
    score = torch.where((blk < 1) | (blk >= count - 1), math.inf, score)        # the first and the last one
    score = torch.where(blk < count, score, -math.inf)
    ids = score.sort(dim=-1, descending=True, stable=True).indices[..., :n]
    took = count.clamp(max=n)
    ids = torch.where(torch.arange(ids.shape[-1], device="cuda") < took, ids, most).sort(-1).values
    real = ids < most
    phys = torch.where(real, row.gather(2, ids.clamp(max=most - 1)), -1)
    o = s["out"]
    for x, y in ((o["ids"], torch.where(real, ids, -1)), (o["table"].view(B, hkv, n), phys)):
        x.fill_(-1)
        x[..., :ids.shape[-1]] = y
    tail = lens[:, None, None] - (count - 1) * bs
    o["lens"].copy_(((took - 1) * bs + tail).expand(B, hkv, 1).flatten())
    return o


def _softmax(x):
    e = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-3e38))
    return e / e.sum(-1, keepdim=True).clamp(min=1e-38)


def _plain_decode(s, case):
    B, hq, hkv, r, dv, bs = (case[x] for x in ("batch", "h_q", "h_kv", "r", "d_v", "block"))
    at = torch.arange(case["n_select"] * bs, device="cuda")
    rows = s["pick"].long().clamp(min=0)[:, at // bs] * bs + at % bs            # [B * H, tokens]
    k, v = _keys(s, case, rows), s["v"].view(-1, dv)[rows].float()
    x = s["q"].view(B * hkv, -1, r).float() @ k.transpose(1, 2) * (1 / math.sqrt(r))
    x = x.masked_fill((at >= s["pick_lens"][:, None])[:, None], -math.inf)
    s["out"].copy_((_softmax(x) @ v).view(B, hq, dv))
    return s["out"]


def _plain_weights(s, case):
    B, hkv, r, n = (case[x] for x in ("batch", "h_kv", "r", "queries"))
    lens = s["lens"].long()
    t = torch.arange(case["ctx"], device="cuda")
    rows = _rows(s, case, t.expand(B, 1, -1))
    k = _keys(s, case, rows)
    pos = lens[:, None] - n + torch.arange(n, device="cuda")                    # [B, n]
    seen = t <= pos[..., None]                                                  # a query before the start sees none
    x = s["q"].view(B, hkv, -1, n, r).flatten(2, 3).float() @ k.transpose(2, 3) * (1 / math.sqrt(r))
    x = x.unflatten(2, (-1, n)).masked_fill(~seen[:, None, None], -math.inf)
    p = _softmax(x).sum((2, 3))                                                 # [B, H, ctx]
    w = s["w"].view(-1)
    before = torch.where((t < s["old"].long()[:, None])[:, None], case["decay"] * w[rows], 0.0)
    live = (t < lens[:, None])[:, None].expand(-1, hkv, -1)
    w[rows[live]] = (before + p)[live]
    return s["w"]


def _plain_evict(s, case):
    B, hkv, keep, recent, ctx = (case[x] for x in ("batch", "h_kv", "keep", "recent", "ctx"))
    lens = s["lens"].long()
    t = torch.arange(ctx, device="cuda").expand(B, hkv, -1)
    rows = _rows(s, case, t)
    L = lens[:, None, None]
    cut = L > keep                                              # the others stay as they are
    w = s["w"].view(-1)[rows]
    rank = torch.where(t < L - recent, w, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    best = torch.zeros_like(t, dtype=torch.bool).scatter_(2, rank[..., :keep - recent], True)
    best &= t < L - recent
    hole = ~best & (t < keep - recent) & cut
    move = best & (t >= keep - recent) & cut
    # the i-th moved token goes to the i-th hole
    spot = torch.zeros(B, hkv, ctx + 1, device="cuda", dtype=torch.int64)
    spot.scatter_(2, torch.where(hole, hole.cumsum(2) - 1, ctx), t)
    to = torch.where(move, spot.gather(2, (move.cumsum(2) - 1).clamp(min=0)), t)
    late = (t >= L - recent) & (t < L) & cut
    to = torch.where(late, t - (L - keep), to)
    kept = torch.full((B, hkv, ctx + 1), -1, device="cuda")
    stay = (best | late) & cut | ~cut & (t < L)
    kept.scatter_(2, torch.where(stay, to, ctx), t)
    s["kept"].fill_(-1)
    s["kept"][..., :min(keep, ctx)] = kept[..., :min(keep, ctx)]
    moved = (move | late) & (to != t)
    src, dst = rows[moved], rows.gather(2, to)[moved]
    for x in (s["k"].view(-1, s["k"].shape[-1]), s["v"].view(-1, case["d_v"]),
              None if s["scale_k"] is None else s["scale_k"].view(-1)):
        if x is not None:
            x[dst] = x[src]
    s["w_out"].view(-1)[rows.gather(2, to)[stay]] = w[stay]
    s["lens_out"].copy_(lens.clamp(max=keep))
    return _evicted(s)


# --------------------------------------------------------------------------------------- run

def _evicted(s):
    out = dict(k=s["k"], v=s["v"], w=s["w_out"], lens=s["lens_out"], kept=s["kept"])
    return out if s["scale_k"] is None else dict(out, scale_k=s["scale_k"])


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"bounds": _plain_bounds, "select": _plain_select, "decode": _plain_decode,
                "weights": _plain_weights, "evict": _plain_evict}[op](s, case)
    s["call"]()
    return {"bounds": s.get("bounds"), "select": s.get("out"), "decode": s.get("out"),
            "weights": s.get("w")}[op] if op != "evict" else _evicted(s)


# -------------------------------------------------------------------------------------- work

def work(case):
    B, hq, hkv, r, dv, op = (case[x] for x in ("batch", "h_q", "h_kv", "r", "d_v", "op"))
    ctx = case["ctx"] * (1 if B == 1 else 0.875)                 # mean of the ragged lengths
    pairs = B * hkv
    key = {"bf16": 2 * r, "int8": r + 4, "int4": r // 2 + 4}[case["k"]]
    if op == "bounds":
        new = min(case["new"], ctx)
        tokens = min(ctx, new + case["block"] / 2)               # a touched block is read from its start
        return dict(bytes=pairs * (tokens * key + max(1, tokens / case["block"]) * 4 * r), flops=pairs * tokens * 2 * r)
    if op == "select":
        blocks = max(1, ctx / case["block"])
        return dict(bytes=pairs * (blocks * 4 * r + 8 * min(case["n_select"], blocks)) + 2 * B * hq * r,
                    flops=B * hq * blocks * 4 * r)
    if op == "decode":
        tokens = min(ctx, case["n_select"] * case["block"])
        return dict(bytes=pairs * tokens * (key + 2 * dv) + 2 * B * hq * (r + dv), flops=B * hq * tokens * 2 * (r + dv))
    if op == "weights":
        return dict(bytes=pairs * ctx * (key + (8 if case["decay"] else 4)) + 2 * B * hq * case["queries"] * r,
                    flops=B * hq * case["queries"] * ctx * 2 * r)
    keep, recent = case["keep"], case["recent"]
    if ctx <= keep:
        return dict(bytes=pairs * ctx * 8, flops=0)
    holes = (keep - recent) * (1 - (keep - recent) / max(1, ctx - recent))
    return dict(bytes=pairs * (ctx * 4 + keep * 8 + 2 * (holes + recent) * (key + 2 * dv)), flops=0)


# ------------------------------------------------------------------------------------- exact

def _row_of(s, case, b, g, t):
    ps = case["page"]
    if ps:
        return (s["table"][b].long()[t // ps] * case["h_kv"] + g) * ps + t % ps
    return (b * case["h_kv"] + g) * _capacity(case) + t


def _key64(s, case, rows):
    k = s["k"].reshape(-1, s["k"].shape[-1])[rows]
    if case["k"] == "int4":
        low, high = k.long() % 16, k.long() // 16
        k = torch.stack([low, high], -1).reshape(*k.shape[:-1], -1)
        k = torch.where(k > 7, k - 16, k)
    k = k.double()
    return k if case["k"] == "bf16" else k * s["scale_k"].reshape(-1)[rows].double().unsqueeze(-1)


def _outward64(x, up):
    m, e = torch.frexp(x)
    m = m * 256
    return torch.ldexp(m.ceil() if up else m.floor(), e - 8)


def exact(case, seed):
    """One kv head of one sequence at a time, in 64 bits."""
    op = case["op"]
    if op == "select":
        return None
    s = prepare(case, seed)
    B, hkv, r, dv = (case[x] for x in ("batch", "h_kv", "r", "d_v"))
    G = case["h_q"] // hkv
    lens = s["lens"].tolist()
    flat = {x: s[x].double().reshape(-1, s[x].shape[-1]) for x in ("k", "v") if op == "evict"}
    if op == "evict":
        flat.update({x: s[x].double().reshape(-1) for x in ("w", "w_out")})
        if s["scale_k"] is not None:
            flat["scale_k"] = s["scale_k"].double().reshape(-1)
    elif op == "weights":
        w = s["w"].double().reshape(-1)
    elif op == "bounds":
        box = s["bounds"].double().reshape(-1, 2, r)
    else:
        o = torch.zeros(B, hkv, G, dv, dtype=torch.float64, device="cuda")
    for b in range(B):
        for g in range(hkv):
            L = lens[b]
            t = torch.arange(L, device="cuda")
            if op == "bounds":
                bs, first = case["block"], int(s["old"][b]) // case["block"]
                last = (L - 1) // bs
                k = _key64(s, case, _row_of(s, case, b, g, t[first * bs:]))
                room = (last - first + 1) * bs - k.shape[0]
                lo, hi = (torch.cat([k, k.new_full((room, r), fill)]).view(-1, bs, r) for fill in (math.inf, -math.inf))
                at = _row_of(s, case, b, g, torch.arange(first, last + 1, device="cuda") * bs) // bs
                box[at] = torch.stack([_outward64(lo.min(1).values, False), _outward64(hi.max(1).values, True)], 1)
            elif op == "decode":
                n = int(s["pick_lens"][b * hkv + g])
                t = torch.arange(n, device="cuda")
                rows = s["pick"][b * hkv + g].long()[t // case["block"]] * case["block"] + t % case["block"]
                x = s["q"][b, g * G:(g + 1) * G].double() @ _key64(s, case, rows).T / math.sqrt(r)
                o[b, g] = torch.softmax(x, -1) @ s["v"].reshape(-1, dv)[rows].double()
            elif op == "weights":
                rows = _row_of(s, case, b, g, t)
                n = case["queries"]
                k = _key64(s, case, rows)
                total = torch.where(t < int(s["old"][b]), case["decay"] * w[rows], 0)
                for i in range(max(0, n - L), n):
                    x = s["q"][b, g * G:(g + 1) * G, i].double() @ k[:L - n + i + 1].T / math.sqrt(r)
                    total[:L - n + i + 1] += torch.softmax(x, -1).sum(0)
                w[rows] = total
            else:
                keep, recent = case["keep"], case["recent"]
                rows = _row_of(s, case, b, g, t)
                order = t
                if L > keep:
                    top = torch.argsort(flat["w"][rows[:L - recent]], descending=True, stable=True)[:keep - recent]
                    top = top.sort().values
                    order = torch.full((keep,), -1, device="cuda")
                    stays = top[top < keep - recent]
                    order[stays] = stays
                    order[:keep - recent][order[:keep - recent] < 0] = top[top >= keep - recent]
                    order[keep - recent:] = t[L - recent:]
                for x in flat:
                    if x == "w_out":
                        flat[x][rows[:len(order)]] = flat["w"][rows[order]]
                    elif x != "w":
                        flat[x][rows[:len(order)]] = flat[x][rows[order]].clone()
    if op == "bounds":
        return box.view(s["bounds"].shape)
    if op == "decode":
        return o.view(B, case["h_q"], dv)
    if op == "weights":
        return w.view(s["w"].shape)
    return dict(k=flat["k"].view(s["k"].shape) if case["k"] == "bf16" else None, v=flat["v"].view(s["v"].shape),
                w=flat["w_out"].view(s["w"].shape), lens=None, kept=None,
                **({} if s["scale_k"] is None else dict(scale_k=flat["scale_k"].view(s["scale_k"].shape))))
