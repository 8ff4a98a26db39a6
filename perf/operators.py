"""What is measured of the operators between a projection and the attention: per-head norm and
rotation of queries and keys (forward, backward, and straight into the cache), and the page tables
and slot maps of a paged cache.

A case's ``op`` says which operator it is a pass of:

``norm_rope``     q, k and v as the projection leaves them (one packed row per token) to the
                  head-major tensors that prefill attention reads: RMS norm per head, weight,
                  rotation by the token's positions.
``backward``      its gradients, from head-major gradients to the packed row's, and the weights'.
``append``        the same forward with k and v written to their cache slots.
``block_tables``  pages, slots and positions of the step's new tokens from request lengths.
"""

import math

import torch

own = False

EPS = 1e-6
W_OFFSET = 0.0
BASE = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------- cases

def _qk(name, op, batch, seq, h_q, h_kv, r, d_v, **kw):
    c = dict(name=name, op=op, batch=batch, seq=seq, h_q=h_q, h_kv=h_kv, r=r, d_v=d_v, rot=r,
             layout="half", axes=1, norm=True, x="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # one GPT-2-small prompt: 12 thin heads, rotation only; a few microseconds of work
        _qk("rope_gpt2_prompt_256", "norm_rope", 1, 256, 12, 12, 16, 64, norm=False, out="bf16"),
        # a serving engine's prompt chunk of the Mistral shape, long after the sequence's start
        _qk("norm_rope_mistral_4096", "norm_rope", 1, 4096, 32, 8, 32, 128, out="bf16", start=65536),
        # two clips of 27 x 45 patches a frame, three position axes, neighbouring pairs, fp32 activations
        _qk("norm_rope_video_9721", "norm_rope", 2, 9721, 16, 16, 64, 64, layout="pair", axes=3,
            x="f32", out="bf16"),
        # training forward of the 7B multi-head shape, the largest
        _qk("norm_rope_7b_b2_s8192", "norm_rope", 2, 8192, 32, 32, 32, 128, out="bf16"),
        # full-width keys, fp32 training of a small model with an odd length, half of a head rotated
        _qk("backward_small_f32_333", "backward", 3, 333, 8, 2, 128, 128, rot=64, x="f32", dy="f32"),
        # images: two axes, grouped heads, bf16 gradients
        _qk("backward_image_2047", "backward", 4, 2047, 16, 4, 64, 128, axes=2, layout="pair", dy="bf16"),
        # training backward of the 7B shape: fp32 gradients from the attention's backward
        _qk("backward_7b_b2_s8192", "backward", 2, 8192, 32, 32, 32, 128, dy="f32"),
        # one decode step of 16 sequences over a paged cache: latency
        _qk("append_decode_b16", "append", 16, 1, 32, 8, 32, 128, k="bf16", page=64, ctx=4096),
        # one decode step of many sequences with wider keys
        _qk("append_decode_b509_r128", "append", 509, 1, 16, 2, 128, 128, k="bf16", page=16, ctx=512, rot=64),
        # a prompt of two sequences that fills an int8-key cache
        _qk("append_prompt_int8_4096", "append", 2, 4096, 32, 8, 32, 128, k="int8", page=0, ctx=0),
        # a decode step of 64 requests: one token each, some of them finished
        dict(name="tables_decode_b64", op="block_tables", batch=64, page=64, max_pages=2048, ctx=100000,
             new=1, done=0.05, spare=1.0, per_seq=1),
        # many prompts admitted at once, ragged, packed; the pool holds most of them
        dict(name="tables_prompts_b512", op="block_tables", batch=512, page=16, max_pages=1024, ctx=2000,
             new=8192, done=0.1, spare=0.97, per_seq=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope", "backward", "backward", "append", "append", "block_tables"])
    if op == "block_tables":
        decode = rng.random() < 0.5
        return dict(op=op, batch=_log_int(rng, 1, 1024 if decode else 512), page=rng.choice([16, 32, 64, 128, 256]),
                    max_pages=1024, ctx=_log_int(rng, 16, 8000), new=1 if decode else _log_int(rng, 8, 8192),
                    done=rng.choice([0.0, 0.05, 0.3]), spare=rng.choice([0.5, 0.97, 1.0]),
                    per_seq=1 if decode and rng.random() < 0.5 else 0)
    r = rng.choice([16, 32, 64, 128])
    h_kv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, r=r, h_kv=h_kv, h_q=h_kv * rng.choice([1, 2, 4, 8]), d_v=rng.choice([64, 128]),
             rot=rng.choice([r, r, r, r // 2]), layout=rng.choice(["half", "pair"]), axes=rng.choice([1, 1, 2, 3]),
             norm=rng.random() < 0.8, x=rng.choice(["bf16", "bf16", "f32"]))
    if c["rot"] < 16:
        c["axes"] = 1
    if op == "append":
        c["k"] = rng.choice(["bf16", "bf16", "bf16", "int8", "int8", "int4"] if r >= 32 else ["bf16", "int8"])
        if rng.random() < 0.5 and c["k"] == "bf16":
            c.update(batch=_log_int(rng, 1, 512), seq=1, page=rng.choice([0, 16, 64, 256]), ctx=_log_int(rng, 16, 1024))
        else:
            c.update(batch=rng.choice([1, 2, 3]), seq=_log_int(rng, 2, 4096), page=0 if c["k"] != "bf16" else 64, ctx=0)
        return c
    tokens = _log_int(rng, 1, 16384)
    c["batch"] = rng.choice([1, 2, 3]) if tokens >= 3 else 1
    c["seq"] = max(1, tokens // c["batch"])
    c["out" if op == "norm_rope" else "dy"] = rng.choice(["bf16", "bf16", "f32"] if op == "norm_rope" else ["bf16", "f32"])
    c["start"] = rng.choice([0, 0, 4096, 100000])
    return c


# ------------------------------------------------------------------------------------ inputs

def _rotation(case):
    """Inverse frequency and position axis of each pair: every axis has a run of pairs with
    frequencies of its own, as image and video models lay them out."""
    pairs, axes = case["rot"] // 2, case["axes"]
    runs = [pairs // axes + (1 if a < pairs % axes else 0) for a in range(axes)]
    freq, axis = [], []
    for a, n in enumerate(runs):
        freq += [BASE ** (-i / n) for i in range(n)]
        axis += [a] * n
    return freq, axis


def _positions(case, gen):
    """int32 [axes, batch, seq]: text counts on from a start of each sequence, patches are
    (frame, row, column) or (row, column) of frames of 27 x 45."""
    B, S, n = case["batch"], case["seq"], case["axes"]
    i = torch.arange(S, device="cuda").repeat(B, 1)
    if n == 1:
        top = case.get("start", 0)
        i = i + torch.randint(0, top + 1, (B, 1), device="cuda", generator=gen)
        return i[None].to(torch.int32).contiguous()
    col, row, frame = i % 45, (i // 45) % 27, i // (45 * 27)
    return torch.stack([frame, row, col] if n == 3 else [i // 45, col]).to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "block_tables":
        return _prepare_tables(case, seed, gen, s)
    B, S, hq, hkv, r, dv = (case[x] for x in ("batch", "seq", "h_q", "h_kv", "r", "d_v"))
    dt = DTYPES[case["x"]]
    width = (hq + hkv) * r + hkv * dv

    def heads(packed):
        q, k, v = packed.split([hq * r, hkv * r, hkv * dv], dim=-1)
        return (q.view(B, S, hq, r).transpose(1, 2), k.view(B, S, hkv, r).transpose(1, 2),
                v.view(B, S, hkv, dv).transpose(1, 2))

    # the projection's rows: unit variance times a size of each token's own
    qkv = torch.randn(B, S, width, device="cuda", generator=gen)
    qkv *= torch.exp(0.5 * torch.randn(B, S, 1, device="cuda", generator=gen))
    s["qkv"] = qkv.to(dt)
    s["q"], s["k"], s["v"] = heads(s["qkv"])
    s["wq"] = s["wk"] = None
    if case["norm"]:
        s["wq"] = 1 + 0.2 * torch.randn(r, device="cuda", generator=gen)
        s["wk"] = 1 + 0.2 * torch.randn(r, device="cuda", generator=gen)
    s["pos"] = _positions(case, gen)
    s["freq"], s["axis"] = _rotation(case)
    s["freq_t"] = torch.tensor(s["freq"], device="cuda", dtype=torch.float32)
    s["axis_t"] = torch.tensor(s["axis"], device="cuda", dtype=torch.int64)
    if own:
        from paper_2603_04427_gb300 import binding as tk
        s["plan"] = tk.rope_plan(r, rot_dim=case["rot"], layout=case["layout"], inv_freq=s["freq"],
                                 pair_axis=s["axis"], norm=case["norm"], eps=EPS, w_offset=W_OFFSET)
    if case["op"] == "norm_rope":
        ot = DTYPES[case["out"]]
        s["out"] = (torch.empty(B, hq, S, r, device="cuda", dtype=ot),
                    torch.empty(B, hkv, S, r, device="cuda", dtype=ot),
                    torch.empty(B, hkv, S, dv, device="cuda", dtype=ot))
    elif case["op"] == "backward":
        gt = DTYPES[case["dy"]]
        s["g"] = tuple(torch.randn(B, h, S, w, device="cuda", generator=gen).to(gt)
                       for h, w in ((hq, r), (hkv, r), (hkv, dv)))
        s["dqkv"] = torch.empty_like(s["qkv"])
        s["dq"], s["dk"], s["dv"] = heads(s["dqkv"])
        s["dwq"] = torch.empty(r, device="cuda") if case["norm"] else None
        s["dwk"] = torch.empty(r, device="cuda") if case["norm"] else None
        if own:
            s["ws"] = tk.qk_norm_rope_workspace(s["plan"], device="cuda")
    else:
        _prepare_cache(case, seed, gen, s)
        if own:
            s["call"] = tk.prepare_qk_norm_rope_append(
                s["cache"], s["plan"], s["q"], s["k"], s["v"], s["pos"], s["slots"], s["q_out"],
                q_weight=s["wq"], k_weight=s["wk"])
    return s


def _prepare_cache(case, seed, gen, s):
    B, S, hq, hkv, r, dv = (case[x] for x in ("batch", "seq", "h_q", "h_kv", "r", "d_v"))
    page, kd = case["page"], case["k"]
    # tokens cached before: the last rows of a context for a decode step, none for a prompt
    lens = torch.randint(0, case["ctx"] + 1, (B,), device="cuda", generator=gen)
    cap = (case["ctx"] + S + 15) // 16 * 16
    where = lens[:, None] + torch.arange(S, device="cuda")
    if page:
        per = (case["ctx"] + S + page - 1) // page
        lead = (B * per, hkv, page)
        table = torch.randperm(B * per, device="cuda", generator=gen).view(B, per)
        slots = table.gather(1, where // page) * page + where % page
        s["table"] = table.to(torch.int32)
    else:
        lead = (B, hkv, cap)
        slots = torch.arange(B, device="cuda")[:, None] * cap + where
    s["slots"] = slots.to(torch.int32).contiguous()
    if case["axes"] == 1:
        s["pos"] = where.to(torch.int32)[None].contiguous()
    if kd == "bf16":
        s["kc"] = torch.randn(*lead, r, device="cuda", generator=gen).to(torch.bfloat16)
        s["ks"] = None
    else:
        s["kc"] = torch.zeros(*lead, r if kd == "int8" else r // 2, device="cuda",
                              dtype=torch.int8 if kd == "int8" else torch.uint8)
        s["ks"] = torch.zeros(*lead, device="cuda")
        s["kv"] = torch.empty(*lead, r, device="cuda", dtype=torch.bfloat16)  # the keys' values
        nib = torch.arange(256, device="cuda")
        s["lut"] = torch.stack([(nib % 16 + 8) % 16 - 8, (nib // 16 + 8) % 16 - 8], 1).float()
    s["vc"] = torch.randn(*lead, dv, device="cuda", generator=gen).to(torch.bfloat16)
    s["q_out"] = torch.empty(B, hq, S, r, device="cuda", dtype=torch.bfloat16)
    if own:
        from paper_2603_04427_gb300 import binding as tk
        fmt = {"bf16": tk.TK_BF16, "int8": tk.TK_I8, "int4": tk.TK_I4}[kd]
        desc = tk.tk_cache_desc(B, hq, hkv, r, dv, 0 if page else cap, page, lead[0] if page else 0,
                                s["table"].shape[1] if page else 0, fmt)
        s["cache"] = tk.ThinKeyCache(desc, s["kc"], s["vc"], s["ks"], s.get("table"))


def _token_rows(case):
    """Rows of the slot map: one per request, or a step's budget of packed tokens, a tenth above
    the mean of the requested ones."""
    if case["per_seq"]:
        return case["batch"] * case["per_seq"]
    mean = 1.0 if case["new"] == 1 else (case["new"] - 1) / math.log(case["new"])
    return int(1.1 * case["batch"] * mean) + 1


def _prepare_tables(case, seed, gen, s):
    B, ps, mp = case["batch"], case["page"], case["max_pages"]
    top = min(case["ctx"], mp * ps)
    lens = torch.randint(0, top + 1, (B,), device="cuda", generator=gen)
    if case["new"] == 1:
        new = torch.ones(B, device="cuda", dtype=torch.int64)
    else:  # prompt lengths: spread over their logarithm, some requests idle
        u = torch.rand(B, device="cuda", generator=gen)
        new = torch.exp(u * math.log(case["new"])).round().to(torch.int64)
        new[torch.rand(B, device="cuda", generator=gen) < 0.05] = 0
    new[torch.rand(B, device="cuda", generator=gen) < case["done"]] = -1
    held = (lens + ps - 1) // ps
    need = ((lens + new.clamp(min=0) + ps - 1) // ps - held)
    used = int(held.sum().item())
    P = B * (-(-top // ps) + -(-case["new"] // ps))       # pages of the pool; some belong to others
    spare = min(P - used, int(need.clamp(min=0).sum().item() * case["spare"]))
    ids = torch.randperm(P, device="cuda", generator=gen)
    p = torch.arange(mp, device="cuda")
    first = held.cumsum(0) - held
    table = torch.where(p < held[:, None], ids[(first[:, None] + p).clamp(max=P - 1)], -1)
    free = torch.zeros(P, device="cuda", dtype=torch.int64)
    free[:spare] = ids[used:used + spare]
    T = case["per_seq"]
    s["max_tokens"] = _token_rows(case)
    i32 = dict(device="cuda", dtype=torch.int32)
    s["lens"], s["new"], s["table"], s["free"] = (x.to(torch.int32).contiguous() for x in (lens, new, table, free))
    s["count"] = torch.tensor([spare], **i32)
    s["out"] = dict(lens=torch.empty(B, **i32), count=torch.empty(1, **i32), refused=torch.empty(1, **i32),
                    offsets=torch.empty(B + 1, **i32), slots=torch.empty(s["max_tokens"], **i32),
                    positions=torch.empty(s["max_tokens"], **i32))
    if own:
        from paper_2603_04427_gb300 import binding as tk
        pool = tk.PagePool(ps, s["table"], s["free"], s["count"], s["lens"],
                           torch.zeros(1, **i32))
        o = s["out"]
        s["call"] = tk.prepare_block_tables(
            pool, s["new"], o["slots"], o["positions"], tokens_per_seq=T, offsets=o["offsets"],
            seq_lens_out=o["lens"], free_count_out=o["count"], refused=o["refused"])
    return s


# ------------------------------------------------------------------------------------- plain

def _cos_sin(pos, axis, freq):
    """cos and sin of pos[axis] * freq in 32 bits, [batch, seq, pairs].  A position p = p1 + p0
    (p0 < 512) and a frequency f = f1 + f0 (f1 a multiple of 2^-12) make products p1 f1 and p0 f1
    that 24 bits hold, so the angle loses nothing at large positions; |p f0| is small."""
    p = pos.permute(1, 2, 0)[:, :, axis]
    p0 = p.remainder(512)
    f1 = (freq * 4096).round() / 4096
    a, b, c = (p - p0).float() * f1, p0.float() * f1, p.float() * (freq - f1)
    ca, sa, cb, sb, cc, sc = a.cos(), a.sin(), b.cos(), b.sin(), c.cos(), c.sin()
    ca, sa = ca * cb - sa * sb, sa * cb + ca * sb
    return ca * cc - sa * sc, sa * cc + ca * sc


def _pairs(y, rot, layout):
    if layout == "half":
        return y[..., :rot // 2], y[..., rot // 2:rot]
    return y[..., 0:rot:2], y[..., 1:rot:2]


def _join(a, b, tail, layout):
    y = torch.cat([a, b], -1) if layout == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([y, tail], -1)


def _rotate(y, cos, sin, case):
    a, b = _pairs(y, case["rot"], case["layout"])
    c, n = cos[:, None], sin[:, None]
    return _join(a * c - b * n, a * n + b * c, y[..., case["rot"]:], case["layout"])


def _norm_rope(x, w, cos, sin, case):
    y = x.float()
    if case["norm"]:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * (w + W_OFFSET)
    return _rotate(y, cos, sin, case)


def _norm_rope_backward(x, w, g, cos, sin, case):
    g = _rotate(g.float(), cos, -sin, case)
    if not case["norm"]:
        return g, None
    x = x.float()
    rho = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xhat = x * rho
    dw = (g * xhat).sum((0, 1, 2))
    g = g * (w + W_OFFSET)
    return rho * (g - xhat * (g * xhat).mean(-1, keepdim=True)), dw


def _plain_append(s, case):
    cos, sin = _cos_sin(s["pos"], s["axis_t"], s["freq_t"])
    s["q_out"].copy_(_norm_rope(s["q"], s["wq"], cos, sin, case))
    k = _norm_rope(s["k"], s["wk"], cos, sin, case).transpose(1, 2)        # [B, S, hkv, r]
    rows = s["vc"].shape[2]                                               # slots a block holds
    at = s["slots"].long()
    block, off = at // rows, at % rows
    s["vc"].transpose(1, 2)[block, off] = s["v"].transpose(1, 2).to(torch.bfloat16)
    if case["k"] == "bf16":
        s["kc"].transpose(1, 2)[block, off] = k.to(torch.bfloat16)
        return
    top = 127.0 if case["k"] == "int8" else 7.0
    scale = k.abs().amax(-1) / top
    code = torch.where(scale[..., None] > 0, (k / scale[..., None]).round().clamp(-top, top), 0.0).to(torch.int32)
    if case["k"] == "int4":
        code = code % 16
        code = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    s["kc"].transpose(1, 2)[block, off] = code.to(s["kc"].dtype)
    s["ks"].transpose(1, 2)[block, off] = scale


def _plain_tables(s, case):
    ps, mp, T = case["page"], case["max_pages"], case["per_seq"]
    B, N = case["batch"], s["max_tokens"]
    L, n, table, free, f = s["lens"].long(), s["new"].long(), s["table"], s["free"], s["count"].long()
    done, want = n < 0, n.clamp(min=0)
    fits = ~done & (L + want <= mp * ps) & ((want <= T) if T else (want.cumsum(0) <= N))
    held = (L + ps - 1) // ps
    need = torch.where(fits, (L + want + ps - 1) // ps - held, 0)
    upto = need.cumsum(0)
    back = torch.where(done, held, 0)
    back_upto = back.cumsum(0)
    total = f + back_upto[-1]
    given = fits & ((need == 0) | (upto <= total))
    m = torch.where(given, want, 0)
    taken = torch.where(given & (need > 0), upto, 0).max()

    def returned(i):                       # page i of those that finished requests give back
        b = torch.searchsorted(back_upto, i, right=True).clamp(max=B - 1)
        return table[b, (i - back_upto[b] + back[b]).clamp(0, mp - 1)]

    def stack(i):
        return torch.where(i < f, free[i.clamp(0, free.numel() - 1)], returned((i - f).clamp(min=0)))

    p = torch.arange(mp, device="cuda")
    new_page = given[:, None] & (p >= held[:, None]) & (p < (held + need)[:, None])
    j = (upto - need - held)[:, None] + p
    table_out = torch.where(new_page, stack(total - 1 - j), table)
    i = torch.arange(free.numel(), device="cuda")
    left = torch.clamp(back_upto[-1] - taken, min=0)
    free_out = torch.where((i >= f) & (i < f + left), returned((i - f).clamp(min=0)), free)
    offsets = torch.cat([m.new_zeros(1), m.cumsum(0)])
    t = torch.arange(N, device="cuda")
    if T:
        b, i = t // T, t % T
        real = i < m[b]
    else:
        b = torch.searchsorted(offsets[1:], t, right=True).clamp(max=B - 1)
        i, real = t - offsets[b], t < offsets[-1]
    pos = torch.where(real, L[b] + i, 0)
    slot = torch.where(real, table_out[b, (pos // ps).clamp(max=mp - 1)] * ps + pos % ps, -1)
    i32 = torch.int32
    return dict(table=table_out, free=free_out, lens=torch.where(done, 0, L + m).to(i32),
                count=(total - taken).to(i32).view(1), refused=(~done & ~given).sum().to(i32).view(1),
                offsets=offsets.to(i32), slots=slot.to(i32), positions=pos.to(i32))


# --------------------------------------------------------------------------------------- run

def _key_values(s, case):
    """The cached keys as the values that their codes stand for."""
    if case["k"] == "bf16":
        return s["kc"]
    codes = s["kc"] if case["k"] == "int8" else s["lut"][s["kc"].int()].flatten(-2)
    return torch.mul(codes, s["ks"][..., None], out=s["kv"])


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "block_tables":
        if not own:
            return _plain_tables(s, case)
        s["call"]()
        return dict(s["out"], table=s["table"], free=s["free"])
    if op == "append":
        if own:
            s["call"]()
        else:
            _plain_append(s, case)
        return dict(q=s["q_out"], k=_key_values(s, case), v=s["vc"])
    if own:
        from paper_2603_04427_gb300 import binding as tk
        if op == "norm_rope":
            q, k, v = s["out"]
            tk.tk_qk_norm_rope(s["plan"], s["q"], s["k"], s["v"], s["pos"], q, k, v,
                               q_weight=s["wq"], k_weight=s["wk"])
            return dict(q=q, k=k, v=v)
        gq, gk, gv = s["g"]
        tk.tk_qk_norm_rope_backward(s["plan"], s["q"], s["k"], s["pos"], gq, gk, gv, s["dq"], s["dk"], s["dv"],
                                    q_weight=s["wq"], k_weight=s["wk"], dq_weight=s["dwq"],
                                    dk_weight=s["dwk"], workspace=s["ws"])
        return dict(qkv=s["dqkv"], wq=s["dwq"], wk=s["dwk"])
    cos, sin = _cos_sin(s["pos"], s["axis_t"], s["freq_t"])
    if op == "norm_rope":
        ot = DTYPES[case["out"]]
        return dict(q=_norm_rope(s["q"], s["wq"], cos, sin, case).to(ot),
                    k=_norm_rope(s["k"], s["wk"], cos, sin, case).to(ot), v=s["v"].to(ot, copy=True).contiguous())
    gq, gk, gv = s["g"]
    dq, dwq = _norm_rope_backward(s["q"], s["wq"], gq, cos, sin, case)
    dk, dwk = _norm_rope_backward(s["k"], s["wk"], gk, cos, sin, case)
    dt = DTYPES[case["x"]]
    packed = torch.cat([t.transpose(1, 2).flatten(2).to(dt) for t in (dq, dk, gv)], -1)
    return dict(qkv=packed, wq=dwq, wk=dwk)


# -------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] == "block_tables":
        # lengths in and out, and each row's slot and position
        return dict(bytes=case["batch"] * 16 + _token_rows(case) * 8, flops=0)
    B, S, hq, hkv, r, dv = (case[x] for x in ("batch", "seq", "h_q", "h_kv", "r", "d_v"))
    size = {"bf16": 2, "f32": 4}
    n, qk, v = B * S, (hq + hkv) * r, hkv * dv
    x = size[case["x"]]
    pos = 4 * case["axes"] * n
    if case["op"] == "norm_rope":
        return dict(bytes=n * (qk + v) * (x + size[case["out"]]) + pos, flops=n * qk * (10 if case["norm"] else 6))
    if case["op"] == "backward":
        g = size[case["dy"]]
        return dict(bytes=n * (qk * (g + x + (x if case["norm"] else 0)) + v * (g + x)) + pos,
                    flops=n * qk * (18 if case["norm"] else 6))
    key = {"bf16": 2 * r, "int8": r + 4, "int4": r // 2 + 4}[case["k"]]
    return dict(bytes=n * (x * (qk + v) + 2 * hq * r + hkv * (key + 2 * dv)) + pos + 4 * n,
                flops=n * qk * (10 if case["norm"] else 6))


# ------------------------------------------------------------------------------------- exact

def exact(case, seed):
    """The definition in 64 bits: pairs as complex numbers turned by exp(i position frequency),
    gradients by the chain rule of torch.autograd over that forward."""
    if case["op"] == "block_tables":
        return None
    s = prepare(case, seed)
    f64 = torch.float64
    freq, pos = s["freq_t"].to(f64), s["pos"].to(f64)
    angle = torch.stack([pos[a] * freq[j] for j, a in enumerate(s["axis"])], -1)   # [B, S, pairs]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    rot, half = case["rot"], case["layout"] == "half"

    def forward(x, w):
        y = x
        if case["norm"]:
            y = x / ((x * x).sum(-1, keepdim=True) / case["r"] + EPS).sqrt() * (w + W_OFFSET)
        z = y[..., :rot]
        z = z.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if half else z.unflatten(-1, (rot // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = (z.transpose(-1, -2) if half else z).flatten(-2)
        return torch.cat([z, y[..., rot:]], -1)

    wq, wk = (None if w is None else w.to(f64) for w in (s["wq"], s["wk"]))
    q, k, v = s["q"].to(f64), s["k"].to(f64), s["v"].to(f64)
    if case["op"] == "backward":
        outs = {}
        got = []
        for name, x, w, g in (("wq", q, wq, s["g"][0]), ("wk", k, wk, s["g"][1])):
            x = x.clone().requires_grad_(True)
            params = [x] if w is None else [x, w.requires_grad_(True)]
            grads = torch.autograd.grad(forward(x, w), params, g.to(f64))
            got.append(grads[0].transpose(1, 2).flatten(2))
            outs[name] = None if w is None else grads[1]
        got.append(s["g"][2].to(f64).transpose(1, 2).flatten(2))
        return dict(outs, qkv=torch.cat(got, -1))
    q, k = forward(q, wq), forward(k, wk)
    if case["op"] == "norm_rope":
        return dict(q=q, k=k, v=v.contiguous())
    B, S = case["batch"], case["seq"]
    kc = torch.zeros_like(s["vc"][..., :1]).expand(*s["vc"].shape[:3], case["r"]).to(f64)
    kc = s["kc"].to(f64) if case["k"] == "bf16" else kc.clone()
    vc = s["vc"].to(f64)
    if case["k"] != "bf16":
        top = 127 if case["k"] == "int8" else 7
        step = k.abs().amax(-1, keepdim=True) / top
        k = torch.where(step > 0, torch.clamp(torch.round(k / step), -top, top) * step, 0)
    rows = vc.shape[2]
    at = s["slots"].long().reshape(-1)
    for h in range(case["h_kv"]):
        for cache, new in ((kc, k), (vc, v)):
            flat = cache[:, h].reshape(-1, cache.shape[-1])
            flat[at] = new[:, h].reshape(B * S, -1)
            cache[:, h] = flat.view(-1, rows, cache.shape[-1])
    return dict(q=q, k=kc, v=vc)
