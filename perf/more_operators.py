"""Operators of a serving loop around the paged cache, as a user's program calls them:

* plan: the step's tables from the requests' lengths, on the device: pages given back and handed out, q_start, and each
  new token's sequence, position and slot (awsrc_kv_plan);
* verify: drafted tokens accepted or not against the target's probabilities from given random numbers, and the token
  that follows them (awsrc_verify_drafts);
* quantize: rows to e4m3 codes with one power-of-two scale per 128 columns, in the products' operand order
  (awsrc_fp8_quantize);
* product: activations times weights held that way, the activations quantised in the call (awsrc_fp8_linear): what
  steps with more rows than the packed GEMV takes and prompts go through.

Where ``own`` is false, ``run`` computes them with elementary torch operations; where it is true it calls the library.
Shapes of the products are those of the Qwen2.5 layers in synth/workloads.py, and generic odd ones.
"""
import math

import torch

own = False

E_MIN = -64  # least exponent of a block of 128


def listed():
    return [
        # one decode step of a few users, a token each: all latency
        dict(name="plan_decode", op="plan", seqs=8, page=64, ctx=1500, new=1, kind="decode"),
        # a step of drafts for many users: some rejected tokens go back, up to five come
        dict(name="plan_drafts", op="plan", seqs=256, page=16, ctx=4096, new=5, kind="drafts"),
        # admission of long prompts beside many users, users that have ended, a pool that does not hold all of it
        dict(name="plan_prompts", op="plan", seqs=1000, page=16, ctx=2000, new=2048, kind="mixed"),
        # one user's four drafts, a small vocabulary
        dict(name="verify_one", op="verify", seqs=1, drafts=4, vocab=32000, dtype="f32", pad=0, draft_probs=True,
             ragged=False),
        # many users' drafts, probabilities of both models over a large vocabulary
        dict(name="verify_batch", op="verify", seqs=64, drafts=5, vocab=151936, dtype="f32", pad=0, draft_probs=True,
             ragged=True),
        # drafts looked up in the text, so without probabilities; odd vocabulary, padded bf16 rows
        dict(name="verify_lookup", op="verify", seqs=24, drafts=8, vocab=50257, dtype="bf16", pad=47,
             draft_probs=False, ragged=True),
        # a projection's weights, once per model load
        dict(name="quantize_weights", op="quantize", rows=11008, cols=2048, dtype="f32", pad=0),
        # a chunk's activations, a column slice of a wider projection, odd row count
        dict(name="quantize_chunk", op="quantize", rows=1023, cols=3584, dtype="bf16", pad=1024),
        # one user's token through a wide projection, float32 as the packed products give it: weight bytes
        dict(name="product_one_token", op="product", rows=1, cols=2048, out=11008, dtype="f32"),
        # a step of drafts: too many rows for the packed GEMV, few for a prompt
        dict(name="product_drafts", op="product", rows=40, cols=3584, out=18944, dtype="bf16"),
        # an odd chunk of an odd layer in float32: nothing is a multiple of a tile
        dict(name="product_odd", op="product", rows=333, cols=5000, out=1777, dtype="f32"),
        # prompts of several users
        dict(name="product_prompts", op="product", rows=8192, cols=3584, out=18944, dtype="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["plan", "verify", "quantize", "product", "product"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "plan":
        kind = rng.choice(["decode", "drafts", "mixed"])
        return {"op": op, "seqs": log(1, 1000), "page": rng.choice([16, 32, 64, 128]), "ctx": log(1, 4096),
                "new": 1 if kind == "decode" else rng.randint(2, 9) if kind == "drafts" else log(16, 2048), "kind": kind}
    if op == "verify":
        vocab = log(100, 151936)
        return {"op": op, "seqs": log(1, 64), "drafts": rng.randint(0, 5), "vocab": vocab, "dtype": dtype,
                "pad": rng.choice([0, 0, (-vocab) % 64, 5]), "draft_probs": rng.random() < 0.7, "ragged": rng.random() < 0.7}
    cols, out = rng.choice([(2048, 2048), (2048, 256), (2048, 11008), (11008, 2048), (3584, 512), (3584, 3584),
                            (18944, 3584), (5120, 1024), (log(64, 6000), log(64, 6000))])
    if op == "quantize":
        return {"op": op, "rows": log(1, 8192), "cols": cols, "dtype": dtype, "pad": rng.choice([0, 0, 8, 3])}
    return {"op": op, "rows": log(1, 8192), "cols": cols, "out": out, "dtype": dtype}


# ------------------------------------------------------------------------------------------------------------ inputs


def plan_lengths(case, seed=0):
    """(tokens held, tokens kept, tokens to come) of each sequence: another seed, another order of the same."""
    held, keep, new = same_lengths(case)
    g = torch.Generator()
    g.manual_seed(seed)
    order = torch.randperm(case["seqs"], generator=g)
    return held[order], keep[order], new[order]


def same_lengths(case):
    g = torch.Generator()
    g.manual_seed(1)
    n, kind = case["seqs"], case["kind"]
    held = (case["ctx"] * (0.25 + 0.75 * torch.rand(n, generator=g))).long().clamp(min=1)
    if kind == "decode":
        return held, held, torch.ones(n, dtype=torch.int64)
    if kind == "drafts":  # the last step's drafts, some of them rejected
        return held, (held - (torch.rand(n, generator=g) * case["new"]).long()).clamp(min=0), \
            1 + (torch.rand(n, generator=g) * case["new"]).long()
    role = torch.rand(n, generator=g)
    keep = torch.where(role < 0.06, 0, held)  # ended
    held = torch.where((role >= 0.06) & (role < 0.1), 0, held)  # a slot that waits for a prompt
    keep = torch.minimum(keep, held)
    new = torch.where(held == 0, (case["new"] * (0.25 + 0.75 * torch.rand(n, generator=g))).long().clamp(min=1), 1)
    return held, keep, torch.where((keep == 0) & (held > 0), 0, new)


def row_lengths(case):
    """Rows of each sequence of a verification: its drafts and one."""
    most = case["drafts"]
    return [1 + (most if not case["ragged"] else int(most * (1.0 - 0.75 * ((b * 0.6180339887) % 1.0)) + 0.5))
            for b in range(case["seqs"])]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "plan":
        prepare_plan(s, case, seed, g)
    elif case["op"] == "verify":
        prepare_verify(s, case, g)
    else:
        prepare_matrix(s, case, g)
    return s


def prepare_plan(s, case, seed, g):
    P, n = case["page"], case["seqs"]
    held, keep, new = plan_lengths(case, seed)
    used, want = -(-held // P), -(-(keep + new) // P)
    stride = int(max(used.max(), want.max())) + 2
    # the pool covers the step with a little to spare, in mixed steps not quite
    short = int((want - used).clamp(min=0).sum() // 8) if case["kind"] == "mixed" else -4
    free = max(0, int((want - used).clamp(min=0).sum()) - int((used - want).clamp(min=0).sum()) - short)
    pages = int(used.sum()) + free
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    s["table"] = torch.full((n, stride), -1, dtype=torch.int32, device="cuda")
    first = torch.cumsum(used, 0) - used
    j = torch.arange(stride)
    mine = (j < used[:, None]).cuda()
    s["table"][mine] = order[(first[:, None] + j).cuda()[mine]]
    s["free"] = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    s["free"][:free] = order[pages - free:]
    s["count"] = torch.tensor([free], dtype=torch.int32, device="cuda")
    s["len"], s["keep"], s["new"] = (t.to(torch.int32).cuda() for t in (held, keep, new))
    s["n_tok"] = int(new.sum()) + 3  # rows of the step's arrays: a few more than tokens
    s["q_start"] = torch.empty(n + 1, dtype=torch.int32, device="cuda")
    s["tok_seq"], s["tok_pos"] = (torch.empty(s["n_tok"], dtype=torch.int32, device="cuda") for _ in range(2))
    s["tok_slot"] = torch.empty(s["n_tok"], dtype=torch.int64, device="cuda")
    if own:
        import paper_2608_23144_gb300 as aw
        s["pool"] = aw.awsrc_kv_pool(s["table"], s["len"], s["free"], s["count"], P)
        s["ws"] = aw.awsrc_step_workspace("cuda")


def prepare_verify(s, case, g):
    rows, V, B = row_lengths(case), case["vocab"], case["seqs"]
    n = sum(rows)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # logits of a target and of a smaller model near it
    logits = randn(n, V) * 2.5
    near = torch.softmax(logits + 0.8 * randn(n, V), -1)
    wide = torch.empty(n, V + case["pad"], dtype=dtype, device="cuda")
    s["p"] = wide[:, :V]
    s["p"].copy_(torch.softmax(logits, -1))
    # the drafts are drawn from the smaller model, or are what the text had: often the target's likeliest
    drawn = (near / torch.empty_like(near).exponential_(generator=g)).argmax(-1)
    likely = torch.where(torch.rand(n, generator=g, device="cuda") < 0.7, logits.argmax(-1), drawn)
    s["ids"] = torch.randint(V, (n,), generator=g, device="cuda").to(torch.int32)
    s["ids"][1:] = (drawn if case["draft_probs"] else likely)[:-1]
    s["q"] = None
    if case["draft_probs"]:
        s["q"] = torch.empty(n, V + case["pad"], dtype=dtype, device="cuda")[:, :V]
        s["q"].copy_(near)
    s["u"] = torch.rand(n, generator=g, device="cuda")
    s["r"] = torch.rand(B, generator=g, device="cuda")
    s["row_start"] = torch.tensor([sum(rows[:b]) for b in range(B + 1)], dtype=torch.int32, device="cuda")
    s["kv_len"] = (torch.randint(4096, (B,), generator=g, device="cuda") + case["drafts"] + 1).to(torch.int32)
    s["accepted"], s["keep"] = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
    s["tokens"] = torch.empty(B, case["drafts"] + 1, dtype=torch.int32, device="cuda")
    s["n"] = n
    if own:
        import paper_2608_23144_gb300 as aw
        s["ws"] = aw.awsrc_step_workspace("cuda")


def prepare_matrix(s, case, g):
    M, K = case["rows"], case["cols"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # activations: a few channels are far larger than the others, tokens differ in size
    x = randn(M, K + case.get("pad", 0)) * torch.exp(0.5 * randn(M, 1))
    x[:, ::max(1, K // 8)] *= 12.0
    s["x"] = x.to(dtype)[:, :K]
    if case["op"] == "product":
        w = randn(case["out"], K) * K ** -0.5
        s["y"] = torch.empty(M, case["out"], dtype=dtype, device="cuda")
        if own:
            import paper_2608_23144_gb300 as aw
            s["w8"] = aw.awsrc_fp8_quantize(w)
        else:
            s["w_codes"], s["w_exp"] = quantized(w)
    if own:
        import paper_2608_23144_gb300 as aw
        s["x8"] = aw.awsrc_fp8_matrix(M, K, "cuda")
        s["ws"] = aw.awsrc_step_workspace("cuda")


# ------------------------------------------------------------------------------------------------- the plain forms


def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2608_23144_gb300 as aw
        if op == "plan":
            aw.awsrc_kv_plan(s["pool"], s["keep"], s["new"], s["ws"], q_start=s["q_start"], tok_seq=s["tok_seq"],
                             tok_pos=s["tok_pos"], tok_slot=s["tok_slot"])
            return {k: s[k] for k in ("table", "len", "free", "count", "q_start", "tok_seq", "tok_pos", "tok_slot")}
        if op == "verify":
            aw.awsrc_verify_drafts(s["row_start"], s["ids"], s["p"], s["q"], s["u"], s["r"], s["ws"], kv_len=s["kv_len"],
                                   accepted=s["accepted"], tokens=s["tokens"], keep=s["keep"])
            return {k: s[k] for k in ("accepted", "tokens", "keep")}
        if op == "quantize":
            aw.awsrc_fp8_quantize(s["x"], out=s["x8"])
            return {"codes": s["x8"].codes, "exps": s["x8"].exps}
        return {"y": aw.awsrc_fp8_linear(s["x"], s["w8"], s["x8"], s["ws"], out=s["y"])}
    return {"plan": plain_plan, "verify": plain_verify, "quantize": plain_quantize, "product": plain_product}[op](s)


def plain_plan(s):
    P, n = s["case"]["page"], s["case"]["seqs"]
    table, free, stride = s["table"], s["free"], s["table"].shape[1]
    held = (s["len"].long() + P - 1) // P
    keep, new, count = s["keep"].long(), s["new"].long(), s["count"].long()
    want = (keep + new + P - 1) // P
    need = (want - held).clamp(min=0)
    room = count + (held - want).clamp(min=0).sum()
    fits = ((need == 0) | (need.cumsum(0) <= room)) & (new.cumsum(0) <= s["n_tok"])
    new = torch.where(fits, new, 0)
    want = (keep + new + P - 1) // P
    back, need = (held - want).clamp(min=0), (want - held).clamp(min=0)
    j = torch.arange(stride, device="cuda")
    # pages given back, in order, on top of the stack
    grow = torch.cat((free, free.new_zeros(1)))
    place = count + (back.cumsum(0) - back)[:, None] + j - want[:, None]
    gone = (j >= want[:, None]) & (j < held[:, None])
    grow[torch.where(gone, place, len(free)).flatten()] = table.flatten()
    free.copy_(grow[:-1])
    count = count + back.sum()
    # pages handed out, from the top
    place = count - 1 - (need.cumsum(0) - need)[:, None] - (j - held[:, None])
    come = (j >= held[:, None]) & (j < want[:, None])
    table.copy_(torch.where(come, free[torch.where(come, place, 0)], table))
    s["count"].copy_(count - need.sum())
    s["len"].copy_(keep + new)
    start = torch.cat((new.new_zeros(1), new.cumsum(0)))
    s["q_start"].copy_(start)
    t = torch.arange(s["n_tok"], device="cuda")
    seq = (torch.searchsorted(start, t, right=True) - 1).clamp(max=n - 1)
    pos = keep[seq] + t - start[seq]
    live = t < start[-1]
    page = table[seq, torch.where(live, pos // P, 0)].long()
    s["tok_seq"].copy_(torch.where(live, seq, -1))
    s["tok_pos"].copy_(torch.where(live, pos, -1))
    s["tok_slot"].copy_(torch.where(live, page * P + pos % P, -1))
    return {k: s[k] for k in ("table", "len", "free", "count", "q_start", "tok_seq", "tok_pos", "tok_slot")}


def plain_verify(s):
    start = s["row_start"].long()
    first, last = start[:-1], start[1:] - 1
    n, B, most = s["n"], s["case"]["seqs"], s["case"]["drafts"]
    row = torch.arange(n, device="cuda")
    draft = s["ids"].long().roll(-1)  # the token that row t's probabilities judge
    p = s["p"].gather(1, draft[:, None])[:, 0].double()
    q = 1.0 if s["q"] is None else s["q"].gather(1, draft[:, None])[:, 0].double()
    seq = torch.searchsorted(start, row, right=True) - 1
    stops = ~(s["u"].double() * q < p) | (row == last[seq])
    at = torch.where(stops, row, n)
    stop = torch.full((B,), n, device="cuda").scatter_reduce_(0, seq, at, "amin")
    accepted = stop - first
    rejected = (stop < last)[:, None]
    full = s["p"][stop].double()
    if s["q"] is None:
        weight = full.scatter(1, draft[stop][:, None], 0.0)
    else:
        weight = (full - s["q"][stop].double()).clamp(min=0)
    weight = torch.where(rejected, weight, full)
    weight = torch.where((weight > 0).any(1, keepdim=True), weight, full)
    sums = weight.cumsum(1)
    token = (sums <= s["r"].double()[:, None] * sums[:, -1:]).sum(1)
    i = torch.arange(most + 1, device="cuda")
    drafts = draft[(first[:, None] + i).clamp(max=n - 1)]
    tokens = torch.where(i < accepted[:, None], drafts, torch.where(i == accepted[:, None], token[:, None], -1))
    s["accepted"].copy_(accepted)
    s["tokens"].copy_(tokens)
    s["keep"].copy_(s["kv_len"] - (last - stop))
    return {k: s[k] for k in ("accepted", "tokens", "keep")}


def power(e):
    """2 to whole numbers, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def quantized(x):
    """(codes [rows, blocks, 128], exponents [rows, blocks]); columns are filled up with zeros."""
    M, K = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -K % 128)).view(M, -1, 128)
    m, e = torch.frexp(x.abs().amax(-1))  # 448 = 0.875 * 2^9
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), E_MIN).clamp(min=E_MIN)
    return (x * power(-e)[..., None]).to(torch.float8_e4m3fn), e


def plain_quantize(s):
    codes, e = quantized(s["x"])
    M, B = e.shape
    rows, blocks, tiles = -(-M // 8) * 8, -(-B // 4) * 4, -(-M // 128)
    # blocks of columns outermost; the 16-byte pieces of a row of 128 change places with the row
    c = torch.zeros(rows, B, 8, 16, dtype=torch.uint8, device="cuda")
    c[:M] = codes.view(torch.uint8).view(M, B, 8, 16)
    r = torch.arange(8, device="cuda")
    c = c.view(rows // 8, 8, B, 8, 16)[:, r[:, None], :, r[:, None] ^ r]  # row, piece, group, block, byte
    c = c.permute(3, 2, 0, 1, 4).reshape(B, rows, 128).view(torch.float8_e4m3fn)
    x = torch.zeros(tiles * 128, blocks, dtype=torch.uint8, device="cuda")
    x[:M, :B] = (e + 127).to(torch.uint8)
    x = x.view(tiles, 4, 32, blocks // 4, 4).permute(3, 0, 2, 1, 4).contiguous()
    return {"codes": c, "exps": x}


def plain_product(s):
    K = s["case"]["cols"]

    def values(codes, e):
        return (codes.float() * power(e)[..., None]).flatten(1)[:, :K]

    x, w = values(*quantized(s["x"])), values(s["w_codes"], s["w_exp"])
    return {"y": (x @ w.T).to(s["y"].dtype)}


# ------------------------------------------------------------------------------------------------------------- work


def work(case):
    if case["op"] == "plan":
        P, n = case["page"], case["seqs"]
        held, keep, new = plan_lengths(case)
        moved = int((-(-(keep + new) // P) - -(-held // P)).abs().sum())
        tokens = int(new.sum()) + 3
        return {"bytes": 4 * (4 * n + n + 3) + 8 * moved + 16 * tokens + 4 * n, "flops": 8 * n + 4 * tokens}
    if case["op"] == "verify":
        size, n = (2 if case["dtype"] == "bf16" else 4), sum(row_lengths(case))
        # half of the sequences are taken to reject a draft and read the row of both models
        rows = case["seqs"] * (1.5 if case["draft_probs"] and case["drafts"] else 1)
        return {"bytes": rows * case["vocab"] * size + n * (8 + 2 * size) + case["seqs"] * (20 + 4 * case["drafts"]),
                "flops": 3 * case["seqs"] * case["vocab"]}
    size, M, K = (2 if case["dtype"] == "bf16" else 4), case["rows"], case["cols"]
    blocks = -(-K // 128)
    if case["op"] == "quantize":
        return {"bytes": M * K * size + M * K + M * blocks, "flops": 3 * M * K}
    N = case["out"]
    return {"bytes": M * K * size + N * K + N * blocks + M * N * size, "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------------------------- the definitions


def exact(case, seed):
    """The definitions, sequence by sequence, whole numbers on the host and numbers in 64 bits."""
    if case["op"] == "product" and 2 * case["rows"] * case["cols"] * case["out"] > 8e12:
        return None
    s = prepare(case, seed)
    return {"plan": exact_plan, "verify": exact_verify, "quantize": exact_quantize, "product": exact_product}[case["op"]](s)


def exact_plan(s):
    P, table, free = s["case"]["page"], s["table"].tolist(), s["free"].tolist()
    length, keep, new, count = s["len"].tolist(), s["keep"].tolist(), s["new"].tolist(), s["count"].item()

    def pages(tokens):
        return -(-tokens // P)

    steps = [pages(k + a) - pages(h) for h, k, a in zip(length, keep, new)]
    room, needed, tokens = count - sum(d for d in steps if d < 0), 0, 0
    for b, d in enumerate(steps):
        needed, tokens = needed + max(d, 0), tokens + new[b]
        if (d > 0 and needed > room) or tokens > s["n_tok"]:
            new[b] = 0
    for b, row in enumerate(table):
        for page in row[pages(keep[b] + new[b]):pages(length[b])]:
            free[count], count = page, count + 1
    start, seq, pos, slot = [0], [], [], []
    for b, row in enumerate(table):
        for j in range(pages(length[b]), pages(keep[b] + new[b])):
            count -= 1
            row[j] = free[count]
        for t in range(keep[b], keep[b] + new[b]):
            seq.append(b)
            pos.append(t)
            slot.append(row[t // P] * P + t % P)
        start.append(len(seq))
    behind = [-1] * (s["n_tok"] - len(seq))

    def i32(v):
        return torch.tensor(v, dtype=torch.int32)

    return {"table": i32(table), "len": i32([k + a for k, a in zip(keep, new)]), "free": i32(free),
            "count": i32([count]), "q_start": i32(start), "tok_seq": i32(seq + behind), "tok_pos": i32(pos + behind),
            "tok_slot": torch.tensor(slot + behind, dtype=torch.int64)}


def exact_verify(s):
    start, ids, kv = s["row_start"].tolist(), s["ids"].tolist(), s["kv_len"].tolist()
    u, r = s["u"].tolist(), s["r"].tolist()
    accepted, tokens, keep = [], [], []
    for b in range(len(kv)):
        row, last, got = start[b], start[b + 1] - 1, []
        while row < last:
            x = ids[row + 1]
            if not u[row] * (1.0 if s["q"] is None else float(s["q"][row, x])) < float(s["p"][row, x]):
                break
            got.append(x)
            row += 1
        w = s["p"][row].double()
        if row < last:
            other = torch.zeros_like(w)
            if s["q"] is None:
                other[ids[row + 1]] = math.inf
            else:
                other = s["q"][row].double()
            rest = torch.where(w > other, w - other, 0.0)
            w = rest if float(rest.max()) > 0 else w
        c = w.cumsum(0)
        token = int(torch.searchsorted(c, (c[-1] * r[b]).view(1), right=True))
        accepted.append(len(got))
        keep.append(kv[b] - (last - row))
        tokens.append((got + [token] + [-1] * s["tokens"].shape[1])[:s["tokens"].shape[1]])
    return {k: torch.tensor(v, dtype=torch.int32) for k, v in (("accepted", accepted), ("tokens", tokens), ("keep", keep))}


def two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def e4m3(x):
    """x rounded to the nearest value of 3 fraction bits and exponents from -6 on, ties to even, in 64 bits."""
    _, p = torch.frexp(x)
    step = two_to((p - 4).clamp(min=-9))
    return torch.round(x / step) * step


def blocks_of(x):
    """For each 128 columns: (first, last + 1, exponent per row, values of the codes) in 64 bits."""
    for a in range(0, x.shape[1], 128):
        part = x[:, a:a + 128].double()
        most = part.abs().amax(1)
        e = (most[:, None] > 448 * two_to(torch.arange(E_MIN, 121, device="cuda"))).sum(1) + E_MIN
        yield a, a + part.shape[1], e, e4m3(part * two_to(-e)[:, None])


def exact_quantize(s):
    M, K = s["x"].shape
    rows, blocks = -(-M // 8) * 8, -(-K // 128)
    codes = torch.zeros(blocks, rows, 128, dtype=torch.float64, device="cuda")
    exps = torch.zeros(-(-blocks // 4), -(-M // 128), 32, 4, 4, dtype=torch.uint8, device="cuda")
    r = torch.arange(M, device="cuda")
    for a, b, e, c in blocks_of(s["x"]):
        k = torch.arange(b - a, device="cuda")
        codes[a // 128][r[:, None], (((k // 16)[None] ^ (r % 8)[:, None]) * 16) + k % 16] = c
        exps[a // 512, r // 128, r % 32, r % 128 // 32, a // 128 % 4] = (e + 127).to(torch.uint8)
    return {"codes": codes, "exps": exps}


def exact_product(s):
    x, K = s["x"], s["x"].shape[1]
    if own:
        w = s["w8"].values().double()
    else:
        w = (s["w_codes"].double() * two_to(s["w_exp"])[..., None]).flatten(1)[:, :K]
    y = torch.zeros(x.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    for a, b, e, c in blocks_of(x):
        y += (c * two_to(e)[:, None]) @ w[:, a:b].T
    return {"y": y}
