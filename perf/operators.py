"""The serving operators of a layer between its packed projections, as a user's program calls them:

* append: new keys and values go into a paged cache held in 8 bits (e4m3 codes, one power-of-two scale per block of
  tokens and head), with the position rotation applied to q and k on the way (awsrc_kv_append);
* attention: ragged queries over that cache, causal, one token to whole prompts (awsrc_paged_attention).

Where ``own`` is false, ``run`` computes both with elementary torch operations in 32 bits; where it is true it calls the
library. Head layouts are those of the Qwen2.5 shapes in synth/workloads.py (16/2, 28/4 and 40/8 heads of 128), plus a
generic one without shared heads.
"""
import math

import torch

own = False

E_MIN, E_MAX, E_NAN = -32, 31, -128  # exponents of a block's scale; -128: the block received a non-finite value
ROPE_BASE = 1e6


def listed():
    base = {"ragged": True, "mixed": False, "interleaved": False, "rotary": 128}
    return [
        # one user, one token: the call in a decode loop, all latency
        dict(base, name="append_one_token", op="append", heads=16, kv_heads=2, dim=128, page=64, dtype="bf16", seqs=1,
             new=1, ctx=1530),
        # a decode step of many users with the packed products' float32 outputs
        dict(base, name="append_decode_batch", op="append", heads=28, kv_heads=4, dim=128, page=64, dtype="f32",
             seqs=128, new=1, ctx=4096),
        # fresh prompts of several users
        dict(base, name="append_prompts", op="append", heads=28, kv_heads=4, dim=128, page=64, dtype="bf16", seqs=6,
             new=2048, ctx=0),
        # long chunks that start and end inside a page, small pages
        dict(base, name="append_long_chunk", op="append", heads=40, kv_heads=8, dim=128, page=16, dtype="bf16", seqs=2,
             new=8191, ctx=24005),
        # other rotation: interleaved pairs on half of the head, no shared heads
        dict(base, name="append_small_heads", op="append", heads=12, kv_heads=12, dim=64, page=32, dtype="f32", seqs=5,
             new=333, ctx=100, interleaved=True, rotary=32),
        # one user's decode step, short context, float32 as the packed products give it: all latency
        dict(base, name="decode_one", op="attention", heads=16, kv_heads=2, dim=128, page=64, dtype="f32", seqs=1,
             new=1, ctx=516),
        # a decode step of a batch with ragged contexts
        dict(base, name="decode_batch", op="attention", heads=28, kv_heads=4, dim=128, page=64, dtype="bf16", seqs=64,
             new=1, ctx=8192),
        # one user with a long context: few rows, a long axis
        dict(base, name="decode_long", op="attention", heads=40, kv_heads=8, dim=128, page=128, dtype="f32", seqs=1,
             new=1, ctx=131070),
        # drafted tokens verified together, small pages
        dict(base, name="verify_drafts", op="attention", heads=28, kv_heads=4, dim=128, page=16, dtype="bf16", seqs=16,
             new=5, ctx=3001),
        # fresh prompts of several users
        dict(base, name="prefill_prompts", op="attention", heads=28, kv_heads=4, dim=128, page=64, dtype="bf16", seqs=4,
             new=4096, ctx=0),
        # chunked prefill beside decoding users, long contexts
        dict(base, name="mixed_chunks", op="attention", heads=40, kv_heads=8, dim=128, page=64, dtype="bf16", seqs=4,
             new=1024, ctx=20011, mixed=True),
        # prompts in float32 with small heads that share nothing, after a cached prefix
        dict(base, name="prefill_small_heads", op="attention", heads=12, kv_heads=12, dim=64, page=32, dtype="f32",
             seqs=3, new=701, ctx=300),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    heads, kv_heads, dim = rng.choice([(16, 2, 128), (28, 4, 128), (40, 8, 128), (12, 12, 64), (14, 2, 64)])
    c = {"op": rng.choice(["append", "attention"]), "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "page": rng.choice([16, 32, 64, 128]), "dtype": rng.choice(["bf16", "bf16", "f32"]), "ragged": rng.random() < 0.8,
         "mixed": False, "interleaved": False, "rotary": dim}
    kind = rng.choice(["decode", "drafts", "prompts", "chunks"])
    if c["op"] == "append":
        c["interleaved"] = rng.random() < 0.25
        c["rotary"] = dim if rng.random() < 0.75 else dim // 2
        if kind in ("decode", "drafts"):
            c.update(seqs=log(1, 128), new=1 if kind == "decode" else rng.randint(2, 8), ctx=log(1, 4096))
        else:
            new = log(17, 8191)
            c.update(seqs=rng.randint(1, max(1, min(6, 16384 // new))), new=new, ctx=0 if kind == "prompts" else log(1, 24005))
        return c
    if kind == "decode":
        ctx = log(1, 131070)
        c.update(seqs=min(64, max(1, log(1, max(2, 524288 * 4 // (ctx * kv_heads))))), new=1, ctx=ctx)
        if c["seqs"] * ctx > 524288:
            c["seqs"] = max(1, 524288 // ctx)
    elif kind == "drafts":
        ctx = log(16, 8192)
        c.update(seqs=rng.randint(1, 16), new=rng.randint(2, 9), ctx=ctx)
    elif kind == "prompts":
        new = log(17, 4096)
        c.update(seqs=rng.randint(1, max(1, min(4, 8192 // new))), new=new, ctx=0)
    else:
        new = log(17, 1024)
        c.update(seqs=rng.randint(1, 4), new=new, ctx=log(17, 16384), mixed=rng.random() < 0.5)
    return c


def lengths(case):
    """(new tokens, tokens before them) of each sequence: the first has the case's, the others of a ragged batch less."""
    new, ctx = [], []
    for b in range(case["seqs"]):
        f = 1.0 - 0.75 * ((b * 0.6180339887) % 1.0) if case["ragged"] else 1.0
        g = 1.0 - 0.75 * ((b * 0.7548776662) % 1.0) if case["ragged"] else 1.0
        new.append(1 if case["mixed"] and b % 3 else max(1, int(case["new"] * f)))
        ctx.append(int(case["ctx"] * g))
    return new, ctx


def exponent(amax):
    """The smallest e with amax <= 448 * 2^e, 448 = 0.875 * 2^9."""
    m, x = torch.frexp(amax)
    e = torch.where(amax > 0, x - 9 + (m > 0.875).int(), E_MIN).clamp(min=E_MIN)
    return torch.where(torch.isfinite(amax) & (e <= E_MAX), e, E_NAN)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, KH, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, ctx = lengths(case)
    B, n = case["seqs"], sum(new)
    kv = [a + b for a, b in zip(new, ctx)]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    used = [-(-k // P) for k in kv]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, max(used), dtype=torch.int32, device="cuda")
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u]
        at += u

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # a few channels of the keys and values are far larger than the others, as in real layers
    chan = torch.exp(0.3 * randn(2, KH, D))
    chan[0, :, :2] *= 6.0

    def filled(layout, scale):
        x = randn(*layout) * scale
        e = exponent(x.abs().amax(dim=(2, 3, 4)))
        return (x * torch.exp2(-e.float())[:, :, None, None, None]).to(torch.float8_e4m3fn), e.to(torch.int8)

    k, k_exp = filled((pages, KH, D // 16, P, 16), chan[0].view(1, KH, D // 16, 1, 16))
    v, v_exp = filled((pages, KH, P // 16, D, 16), chan[1].view(1, KH, 1, D, 1))
    s = {"case": case, "k_cache": k, "v_cache": v, "k_exp": k_exp, "v_exp": v_exp, "table": table, "n": n,
         "q_start": torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda"),
         "kv_len": torch.tensor(kv, dtype=torch.int32, device="cuda"), "max_new": max(new), "max_kv": max(kv)}
    # q, k and v as one projection's output leaves them: rows of all heads
    if case["op"] == "append":
        qkv = randn(n, (H + 2 * KH), D)
        qkv[:, H:H + KH] *= chan[0]
        qkv[:, H + KH:] *= chan[1]
        qkv = qkv.to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
        r = case["rotary"]
        freq = ROPE_BASE ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
        ang = torch.arange(max(kv), device="cuda", dtype=torch.float64)[:, None] * freq
        s["cos"], s["sin"] = ang.cos().float(), ang.sin().float()
        s["out"] = torch.empty(n, H, D, dtype=dtype, device="cuda")
    else:
        s["q"] = randn(n, H, D).to(dtype)
        s["sm_scale"] = D ** -0.5
        s["out"] = torch.empty(n, H, D, dtype=dtype, device="cuda")
        s["lse"] = torch.empty(n, H, dtype=torch.float32, device="cuda")
    if own:  # what a serving program keeps: the cache's and the step's handles and the workspace
        import paper_2608_23144_gb300 as aw
        s["cache"] = aw.awsrc_kv_cache(k, v, k_exp, v_exp)
        s["batch"] = aw.awsrc_kv_batch(s["q_start"], s["kv_len"], table, n, s["max_new"], s["max_kv"])
        s["ws"] = aw.awsrc_attention_workspace(s["cache"], H)
    return s


def run(s):
    if own:
        import paper_2608_23144_gb300 as aw
        if s["case"]["op"] == "append":
            aw.awsrc_kv_append(s["cache"], s["batch"], s["q"], s["k"], s["v"], s["cos"], s["sin"], s["ws"],
                               interleaved=s["case"]["interleaved"], q_out=s["out"])
            return {"q": s["out"], "k": s["k_cache"], "v": s["v_cache"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}
        aw.awsrc_paged_attention(s["cache"], s["batch"], s["q"], s["ws"], sm_scale=s["sm_scale"], out=s["out"],
                                 lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    return plain_append(s) if s["case"]["op"] == "append" else plain_attention(s)


def token_places(s):
    """For each new token: its sequence, its place among the sequence's new tokens and its position."""
    q_start = s["q_start"].long()
    new = q_start[1:] - q_start[:-1]
    seq = torch.repeat_interleave(torch.arange(len(new), device="cuda"), new, output_size=s["n"])
    i = torch.arange(s["n"], device="cuda") - q_start[seq]
    return seq, i, (s["kv_len"].long() - new)[seq] + i


def rotated(x, cos, sin, interleaved):
    x = x.float()
    h = cos.shape[-1]
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :h], x[..., h:2 * h]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, x[..., 2 * h:]), dim=-1)


def plain_append(s):
    P, D = s["case"]["page"], s["case"]["dim"]
    seq, i, pos = token_places(s)
    page, row = s["table"].long()[seq, pos // P], pos % P
    cos, sin = s["cos"][pos], s["sin"][pos]
    q = rotated(s["q"], cos, sin, s["case"]["interleaved"]).to(s["q"].dtype)
    new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    ctx = s["kv_len"].long() - new
    first = s["table"].long().gather(1, (ctx // P)[:, None])[:, 0]  # the page that a sequence's first new token goes to
    older = torch.arange(P, device="cuda")[None] < (ctx % P)[:, None]  # its rows that hold earlier tokens

    def put(x, codes, exps, is_k):
        raw = codes.view(torch.uint8)
        need = torch.zeros(exps.shape, device="cuda").scatter_reduce_(
            0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")[page]
        e = exponent(need).int()  # of each new token's block, from the new tokens alone
        old = exps.int()[first]
        held = (ctx % P > 0)[:, None]
        mine = (page == first[seq])[:, None] & held[seq]
        bad = (e == E_NAN) | (mine & (old[seq] == E_NAN))
        e = torch.where(bad, E_NAN, torch.where(mine, torch.maximum(e, old[seq]), e))
        # the older tokens of the first page, in the block's new scale
        e0 = e[s["q_start"][:-1].long()]
        step = torch.where(held & (e0 != E_NAN) & (old != E_NAN), (old - e0).float(), 0.0).exp2()
        block = raw[first].view(torch.float8_e4m3fn).float() * step[:, :, None, None, None]
        block = block.to(torch.float8_e4m3fn).view(torch.uint8)
        keep = older[:, None, None, :, None] if is_k else older.view(-1, 1, P // 16, 1, 16)
        raw[first] = torch.where(keep, block, raw[first])
        y = torch.where((e == E_NAN)[..., None], 0.0, x * torch.exp2(-e.float())[..., None])
        y = y.to(torch.float8_e4m3fn).view(torch.uint8)
        if is_k:
            raw[page, :, :, row] = y.view(y.shape[0], y.shape[1], D // 16, 16)
        else:
            raw[page, :, row // 16, :, row % 16] = y
        exps[page] = e.to(torch.int8)

    put(rotated(s["k"], cos, sin, s["case"]["interleaved"]), s["k_cache"], s["k_exp"], True)
    put(s["v"].float(), s["v_cache"], s["v_exp"], False)
    return {"q": q, "k": s["k_cache"], "v": s["v_cache"], "k_exp": s["k_exp"], "v_exp": s["v_exp"]}


def scale_of(e):
    return torch.where(e == E_NAN, float("nan"), torch.exp2(e.float()))


def plain_attention(s):
    c = s["case"]
    H, KH, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    seq, i, _ = token_places(s)
    table = s["table"].long()
    B, L, N = table.shape[0], s["max_new"], table.shape[1] * P
    k = s["k_cache"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()  # B, pages, KH, D/16, P, 16
    k = (k * scale_of(s["k_exp"][table])[..., None, None, None]).permute(0, 2, 1, 4, 3, 5).reshape(B, KH, 1, N, D)
    v = s["v_cache"].view(torch.uint8)[table].view(torch.float8_e4m3fn).float()  # B, pages, KH, P/16, D, 16
    v = (v * scale_of(s["v_exp"][table])[..., None, None, None]).permute(0, 2, 1, 3, 5, 4).reshape(B, KH, 1, N, D)
    q = torch.zeros(B, L, H, D, device="cuda")
    q[seq, i] = s["q"].float()
    q = q.view(B, L, KH, H // KH, D).permute(0, 2, 3, 1, 4)
    x = (q @ k.transpose(-1, -2)).mul_(s["sm_scale"])  # B, KH, H/KH, L, N
    new = s["q_start"][1:] - s["q_start"][:-1]
    last = (s["kv_len"] - new)[:, None] + torch.arange(L, device="cuda")  # the last position a query sees
    sees = torch.arange(N, device="cuda") <= torch.minimum(last, s["kv_len"][:, None] - 1)[..., None]
    x.masked_fill_(~sees[:, None, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(torch.isinf(m), 0.0, m)).exp_()
    t = x.sum(-1, keepdim=True)
    out = torch.where(t > 0, (x @ v) / t, 0.0).permute(0, 3, 1, 2, 4).reshape(B, L, H, D)
    lse = (m + t.log()).permute(0, 3, 1, 2, 4).reshape(B, L, H)
    return {"out": out[seq, i].to(s["q"].dtype), "lse": lse[seq, i]}


def work(case):
    H, KH, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    size = 2 if case["dtype"] == "bf16" else 4
    new, ctx = lengths(case)
    n, kv = sum(new), [a + b for a, b in zip(new, ctx)]
    index = 4 * sum(-(-k // P) for k in kv) + 8 * len(new)
    if case["op"] == "append":
        blocks = sum(-(-k // P) - c // P for k, c in zip(kv, ctx))
        rows = len({p for k, c in zip(kv, ctx) for p in range(c, k)})  # distinct rows of the two tables
        return {"bytes": n * (2 * H + 2 * KH) * D * size + 2 * n * KH * D + 2 * blocks * KH + 4 * rows * case["rotary"]
                + 4 * blocks + 8 * len(new), "flops": 3 * n * (H + KH) * case["rotary"] + 2 * n * KH * D}
    pairs = sum(a * c + a * (a + 1) // 2 for a, c in zip(new, ctx))
    return {"bytes": 2 * sum(kv) * KH * D + 2 * sum(-(-k // P) for k in kv) * KH + 2 * n * H * D * size + 4 * n * H + index,
            "flops": 4 * pairs * H * D}


def e4m3(x):
    """x rounded to the nearest value of 3 fraction bits and exponents from -6 on, ties to even, in 64 bits."""
    _, p = torch.frexp(x)
    step = torch.exp2((p - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def exact(case, seed):
    """The definition in 64 bits, sequence by sequence."""
    s = prepare(case, seed)
    H, KH, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, ctx = lengths(case)
    table = s["table"].tolist()
    if case["op"] == "append":
        h = case["rotary"] // 2
        pos = torch.cat([torch.arange(c, c + a) for a, c in zip(new, ctx)]).cuda()
        turn = torch.complex(s["cos"].double()[pos], s["sin"].double()[pos])[:, None]
        dims = torch.arange(2 * h, device="cuda").view(h, 2) if case["interleaved"] else torch.arange(2 * h, device="cuda").view(2, h).T

        def turned(x):
            x = x.double().clone()
            z = torch.complex(x[..., dims[:, 0]], x[..., dims[:, 1]]) * turn
            x[..., dims[:, 0]], x[..., dims[:, 1]] = z.real, z.imag
            return x

        # [page, head, row, dim] in 64 bits
        kc = s["k_cache"].double().permute(0, 1, 3, 2, 4).reshape(-1, KH, P, D)
        vc = s["v_cache"].double().permute(0, 1, 2, 4, 3).reshape(-1, KH, P, D)
        exps = {"k": s["k_exp"].long(), "v": s["v_exp"].long()}
        for key, cache, x in (("k", kc, turned(s["k"])), ("v", vc, s["v"].double())):
            at = 0
            for b in range(len(new)):
                p, end = ctx[b], ctx[b] + new[b]
                while p < end:
                    upto, page, row = min(end, (p // P + 1) * P), table[b][p // P], p % P
                    part = x[at:at + upto - p].transpose(0, 1)  # head, token, dim
                    most = part.abs().amax(dim=(1, 2))
                    e = (most[:, None] > 448 * 2.0 ** torch.arange(E_MIN, E_MAX, device="cuda")).sum(1).double() + E_MIN
                    if row:
                        o = exps[key][page].double()
                        e = torch.maximum(e, o)
                        cache[page, :, :row] = e4m3(cache[page, :, :row] * torch.exp2(o - e)[:, None, None])
                    cache[page, :, row:row + upto - p] = e4m3(part * torch.exp2(-e)[:, None, None])
                    exps[key][page] = e.long()
                    at, p = at + upto - p, upto
        return {"q": turned(s["q"]), "k": kc.view(-1, KH, P, D // 16, 16).permute(0, 1, 3, 2, 4).contiguous(),
                "v": vc.view(-1, KH, P // 16, 16, D).permute(0, 1, 2, 4, 3).contiguous(),
                "k_exp": exps["k"].to(torch.int8), "v_exp": exps["v"].to(torch.int8)}
    out = torch.empty(s["n"], H, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["n"], H, dtype=torch.float64, device="cuda")
    at = 0
    for b in range(len(new)):
        pages = table[b][:-(-(new[b] + ctx[b]) // P)]
        for h in range(KH):
            k = s["k_cache"][pages, h].double() * torch.exp2(s["k_exp"][pages, h].double())[:, None, None, None]
            v = s["v_cache"][pages, h].double() * torch.exp2(s["v_exp"][pages, h].double())[:, None, None, None]
            k = k.transpose(1, 2).reshape(-1, D)[:new[b] + ctx[b]]
            v = v.transpose(2, 3).reshape(-1, D)[:new[b] + ctx[b]]
            for q0 in range(0, new[b], 1024):
                q1, G = min(new[b], q0 + 1024), H // KH
                q = s["q"][at + q0:at + q1, h * G:(h + 1) * G].double()
                x = torch.einsum("ihd,jd->hij", q, k) * s["sm_scale"]
                hidden = torch.arange(len(k), device="cuda")[None] > torch.arange(ctx[b] + q0, ctx[b] + q1, device="cuda")[:, None]
                x = x.masked_fill(hidden, -math.inf)
                lse[at + q0:at + q1, h * G:(h + 1) * G] = torch.logsumexp(x, -1).T
                out[at + q0:at + q1, h * G:(h + 1) * G] = torch.einsum("hij,jd->ihd", torch.softmax(x, -1), v)
        at += new[b]
    return {"out": out, "lse": lse}
