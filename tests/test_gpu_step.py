"""GPU parity of awsrc_kv_plan and awsrc_verify_drafts: every output equal to the
definitions on the host (tests/step_ref.py), and the serving step they belong to."""
import math
import random

import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu

I32 = torch.int32


@pytest.fixture(scope="module")
def aw():
    import paper_2608_23144_gb300 as aw
    assert torch.cuda.is_available()
    return aw


def cuda_ints(v, dtype=I32):
    return torch.tensor(v, dtype=dtype).cuda()


# --------------------------------------------------------------------- plan


class Pool:
    """A pool on the host and on the device; step() runs both and compares everything."""

    def __init__(self, aw, rng, n_seq, page, stride, lengths, spare):
        self.aw, self.page = aw, page
        used = [-(-k // page) for k in lengths]
        pages = list(range(sum(used) + spare))
        rng.shuffle(pages)
        self.table = [[-1] * stride for _ in range(n_seq)]
        at = 0
        for b, k in enumerate(used):
            self.table[b][:k] = pages[at:at + k]
            at += k
        self.free = pages[at:] + [-1] * at
        self.count, self.length = len(pages) - at, list(lengths)
        self.ws = aw.awsrc_step_workspace()
        self.pool = aw.awsrc_kv_pool(cuda_ints(self.table).view(n_seq, stride), cuda_ints(self.length), cuda_ints(self.free),
                                     cuda_ints([self.count]), page)

    def step(self, keep, add, n_tok, maps=True):
        want = ref.plan(self.page, self.table, self.length, self.free, self.count, keep, add, n_tok)
        self.table, self.length, self.free, self.count, q_start, *toks, flags = want
        got = [torch.full((n_tok,), 77, dtype=t, device="cuda") for t in (I32, I32, torch.int64)] if maps else [None] * 3
        q = self.aw.awsrc_kv_plan(self.pool, None if keep is None else cuda_ints(keep), cuda_ints(add), self.ws, n_tok=n_tok,
                                  tok_seq=got[0], tok_pos=got[1], tok_slot=got[2])
        p = self.pool
        assert q.tolist() == q_start
        assert p.kv_len.tolist() == self.length and p.free_count.item() == self.count
        assert p.page_table.tolist() == self.table and p.free_pages.tolist() == self.free
        if maps:
            assert [t.tolist() for t in got] == toks
        assert self.aw.awsrc_workspace_status(self.ws) == flags
        return flags


@pytest.mark.parametrize("n_seq,page,most", [(1, 16, 70), (7, 16, 200), (33, 32, 500), (100, 64, 300), (1000, 128, 600),
                                             (1025, 16, 90), (3000, 16, 40)])
def test_plan_follows_the_definition(aw, n_seq, page, most):
    """Steps of decoding, drafts that go back, ended sequences, prompts, with room for all and without, rows of the step
    fewer and more than the tokens."""
    rng = random.Random(n_seq * 1000 + page)
    lengths = [rng.choice([0, 1, page, page + 1, rng.randrange(most)]) for _ in range(n_seq)]
    pool = Pool(aw, rng, n_seq, page, -(-2 * most // page) + 2, lengths, spare=n_seq // 2 + 3)
    seen = set()
    for kind in ("decode", "drafts", "end", "prompts", "few rows", "decode", "drain", "prompts"):
        add, keep = [1] * n_seq, list(pool.length)
        n_tok = None
        if kind == "drafts":
            keep = [max(0, k - rng.randrange(6)) for k in keep]
            add = [rng.randrange(7) for _ in keep]
        elif kind == "end":
            keep = [0 if rng.random() < 0.4 else k for k in keep]
            add = [0 if k == 0 else 1 for k in keep]
        elif kind == "prompts":
            add = [rng.randrange(most) if k == 0 else 1 for k in keep]
        elif kind == "few rows":
            add = [rng.randrange(4) for k in keep]
            n_tok = max(1, sum(add) * 2 // 3)
        elif kind == "drain":
            keep, add = [0] * n_seq, [0] * n_seq
        seen.add(pool.step(None if kind == "decode" else keep, add, sum(add) + 2 if n_tok is None else n_tok))
    assert 0 in seen and (16 in seen or n_seq < 7)


def test_plan_of_long_prompts(aw):
    rng = random.Random(3)
    pool = Pool(aw, rng, 40, 16, 700, [rng.randrange(3000) for _ in range(40)], spare=20000)
    assert pool.step(None, [rng.randrange(8000) for _ in range(40)], 40 * 8000) == 0
    assert pool.step([0] * 40, [1] * 40, 40) == 0


def test_plan_without_maps_or_sequences(aw):
    rng = random.Random(1)
    pool = Pool(aw, rng, 5, 32, 9, [3, 0, 32, 33, 64], spare=4)
    assert pool.step(None, [1] * 5, 5, maps=False) == 0
    none = aw.awsrc_kv_pool(torch.empty(0, 3, dtype=I32, device="cuda"), cuda_ints([]), cuda_ints([2, 1, 0]), cuda_ints([3]), 64)
    slot = torch.zeros(4, dtype=torch.int64, device="cuda")
    q = aw.awsrc_kv_plan(none, None, cuda_ints([]), pool.ws, tok_slot=slot)
    assert q.tolist() == [0] and slot.tolist() == [-1] * 4 and none.free_count.item() == 3
    assert aw.awsrc_kv_plan(none, None, cuda_ints([]), pool.ws, n_tok=0).tolist() == [0]


@pytest.mark.parametrize("field,value", [("len", -1), ("len", 16 * 9 + 1), ("len", 2 ** 31 - 1), ("keep", -1), ("keep", 41),
                                         ("add", -1), ("add", 2 ** 31 - 1), ("add", 16 * 9 - 39)])
def test_plan_leaves_wrong_entries_alone(aw, field, value):
    rng = random.Random(9)
    pool = Pool(aw, rng, 4, 16, 9, [20, 40, 0, 17], spare=9)
    keep, add = list(pool.length), [1, 1, 20, 1]
    if field == "len":
        pool.length[1] = keep[1] = value
        pool.pool.kv_len[1] = value
    elif field == "keep":
        keep[1] = value
    else:
        add[1] = value
    assert pool.step(keep, add, 100) == 8
    keep = list(pool.length)
    keep[1] = max(0, min(keep[1], 16 * 9))
    if field != "len":
        assert pool.step(keep, [1] * 4, 100) == 0  # the sequence goes on


@pytest.mark.parametrize("count", [-1, 13, 12])
def test_plan_refuses_a_stack_that_cannot_be_right(aw, count):
    """A count outside the stack, or pages that come back twice: nothing changes."""
    rng = random.Random(2)
    pool = Pool(aw, rng, 2, 16, 6, [70, 30], spare=5)  # 12 pages
    pool.count = count
    pool.pool.free_count.fill_(count)
    assert pool.step([0, 30], [0, 1], 3) == 8


# -------------------------------------------------------------- verification


def rows_of(rng, gen, n, vocab, kind, dtype):
    x = torch.randn(n, vocab, generator=gen, dtype=torch.float64) * (6.0 if kind == "sharp" else 1.0)
    p = torch.softmax(x, -1)
    q = torch.softmax(x + torch.randn(n, vocab, generator=gen, dtype=torch.float64), -1)
    if kind == "cut":  # as top-k filters leave them: most are 0
        p = torch.where(p >= p.quantile(0.7, -1, keepdim=True), p, 0.0)
        p /= p.sum(-1, keepdim=True)
    if kind == "same":
        q = p.clone()
    return p.to(dtype), q.to(dtype)


def check(aw, starts, ids, p, q, u, r, max_draft, kv_len, flags=0, pad=0):
    dev_p, dev_q = (None if t is None else torch.nn.functional.pad(t, (pad, 3)).cuda()[:, pad:pad + t.shape[1]] for t in (p, q))
    ws = aw.awsrc_step_workspace()
    n = len(starts) - 1
    keep = torch.full((n,), 99, dtype=I32, device="cuda")
    acc, tok = aw.awsrc_verify_drafts(cuda_ints(starts), cuda_ints(ids), dev_p, dev_q, u.cuda(), r.cuda(), ws,
                                      max_draft=max_draft, kv_len=cuda_ints(kv_len), keep=keep)
    want = ref.verify(starts, ids, p.double().tolist(), None if q is None else q.double().tolist(), u.tolist(), r.tolist(),
                      max_draft, kv_len)
    assert acc.tolist() == want[0]
    assert tok.tolist() == want[1]
    assert keep.tolist() == want[2]
    assert aw.awsrc_workspace_status(ws) == want[3] == flags
    return want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 31, 257, 1000, 4099])
@pytest.mark.parametrize("kind", ["wide", "sharp", "cut", "same", "looked up"])
def test_verify_follows_the_definition(aw, dtype, vocab, kind):
    rng = random.Random(vocab * 10 + len(kind))
    gen = torch.Generator().manual_seed(vocab)
    drafts = [0, 1, 5, 0, 3, 7, 2, 4, 1, 6]
    lens = [d + 1 for d in drafts]
    lens[3] = 0  # a sequence without rows
    starts = [sum(lens[:b]) for b in range(len(lens) + 1)]
    n = starts[-1] + 2  # rows behind the last sequence
    p, q = rows_of(rng, gen, n, vocab, kind, dtype)
    ids = [rng.randrange(vocab) for _ in range(n)]
    for t in range(n - 1):
        if rng.random() < 0.8:
            ids[t + 1] = int(p[t].argmax())
    u, r = torch.rand(n, generator=gen) * rng.choice([1.0, 0.3]), torch.rand(len(drafts), generator=gen)
    r[0], r[1], r[2] = 0.0, 1.0 - 2.0 ** -24, 0.5
    want = check(aw, starts, ids, p, None if kind == "looked up" else q, u, r, 7, [rng.randrange(20, 900) for _ in lens],
                 pad=rng.choice([0, 1, 8]))
    if vocab > 100 and kind in ("wide", "looked up"):  # wide rows: a likeliest token has little of them
        assert any(a < d for a, d in zip(want[0], drafts))  # some were not accepted


@pytest.mark.parametrize("n_seq", [76, 77, 152, 153, 304, 305, 700])
def test_verify_many_sequences(aw, n_seq):
    """Eight thread blocks a sequence down to one, as the number of sequences grows."""
    rng, gen = random.Random(n_seq), torch.Generator().manual_seed(n_seq)
    vocab = 700
    lens = [rng.randrange(0, 3) for _ in range(n_seq)]  # no rows, none drafted, one drafted
    starts = [sum(lens[:b]) for b in range(n_seq + 1)]
    n = starts[-1]
    p, q = rows_of(rng, gen, n, vocab, "wide", torch.float32)
    ids = [rng.randrange(vocab) for _ in range(n)]
    check(aw, starts, ids, p, q, torch.rand(n, generator=gen), torch.rand(n_seq, generator=gen), 1,
          [rng.randrange(20, 900) for _ in lens])


def test_verify_many_drafts_and_a_large_vocabulary(aw):
    gen = torch.Generator().manual_seed(8)
    vocab, drafts = 60001, 70
    p = torch.softmax(torch.randn(drafts + 1, vocab, generator=gen) * 3, -1)
    ids = [0] + p[:-1].argmax(-1).tolist()
    for stop in (0, 31, 32, 33, 69, 70):
        u = torch.zeros(drafts + 1)
        u[stop:] = 0.999
        check(aw, [0, drafts + 1], ids, p, None, u, torch.rand(1, generator=gen), drafts, [500])


def test_verify_places_every_threshold(aw):
    """r at and beside the running sums of weights that are multiples of 2^-10: the token changes exactly there."""
    w = torch.tensor([0, 3, 0, 5, 1, 0, 0, 7, 1008], dtype=torch.float64) / 1024
    sums = w.cumsum(0).float()
    r = torch.cat([sums[:-1], torch.nextafter(sums[:-1], torch.zeros(8)), torch.nextafter(sums[:-1], torch.ones(8))]).clamp(min=0)
    n = len(r)
    p = w.float().repeat(n, 1)
    for q in (None, torch.zeros(n, 9)):
        check(aw, list(range(n + 1)), [0] * n, p, q, torch.rand(n), r, 0, [5] * n)


def test_verify_rows_that_leave_nothing(aw):
    """p below q everywhere (p itself takes over), rows of zeros (no token), a draft that holds all of p, and values that are
    no probabilities."""
    p = torch.zeros(12, 40)
    p[:, 7], p[:, 9] = 0.25, 0.5
    q = p.clone()
    q[2:4] = 1.0
    p[4:6] = 0.0
    p[6], q[6] = 0.0, 0.5
    p[6, 3] = 1.0
    p[8, :20], q[8, :20] = math.nan, 0.0
    p[8, 30] = -3.0
    p[10, 5], p[10, 6] = math.inf, 2.0
    q[10, 5], q[10, 6] = math.nan, -1.0
    ids = [3] * 12
    u, r = torch.full((12,), 0.9999), torch.full((6,), 0.7)
    for draft in (q, None):
        check(aw, [0, 2, 4, 6, 8, 10, 12], ids, p, draft, u, r, 1, [50] * 6)
    u = torch.tensor([math.nan, 0.0, -1.0, 0.0, math.inf, 0.0] + [1.0] * 6)
    r = torch.tensor([math.nan, -1.0, 1.0, math.inf, 0.0, 1e-40])
    check(aw, [0, 2, 4, 6, 8, 10, 12], ids, p, q, u, r, 1, [50] * 6)


@pytest.mark.parametrize("starts,ids,flags", [([0, 3, 2, 4], [1] * 6, 8), ([-1, 2, 4, 6], [1] * 6, 8), ([0, 2, 4, 7], [1] * 6, 8),
                                              ([0, 6, 6, 6], [1] * 6, 8), ([0, 2, 4, 6], [1, -1, 1, 1, 1, 50], 8),
                                              ([0, 0, 0, 0], [1] * 6, 0)])
def test_verify_reports_what_cannot_be_right(aw, starts, ids, flags):
    gen = torch.Generator().manual_seed(1)
    p = torch.softmax(torch.randn(6, 50, generator=gen), -1)
    check(aw, starts, ids, p, None, torch.rand(6, generator=gen), torch.rand(3, generator=gen), 3, [9, 8, 7], flags)


def test_verify_keep_may_be_kv_len_and_may_be_left_out(aw):
    gen = torch.Generator().manual_seed(4)
    p = torch.softmax(torch.randn(8, 300, generator=gen) * 4, -1).cuda()
    ws, starts = aw.awsrc_step_workspace(), cuda_ints([0, 3, 8])
    ids, u, r = cuda_ints([5] * 8), torch.full((8,), 0.5).cuda(), torch.rand(2, generator=gen).cuda()
    kv = cuda_ints([10, 20])
    acc, tok = aw.awsrc_verify_drafts(starts, ids, p, None, u, r, ws, max_draft=4, kv_len=kv, keep=kv)
    acc2, tok2 = aw.awsrc_verify_drafts(starts, ids, p, None, u, r, ws, max_draft=4)
    assert torch.equal(acc, acc2) and torch.equal(tok, tok2)
    assert kv.tolist() == [10 - 2 + acc[0].item(), 20 - 4 + acc[1].item()]


# --------------------------------------------------------- a run of them


def test_a_serving_loop_on_the_device(aw):
    """Prompts, then rounds of drafts as one captured graph: plan, 8-bit q, k, v products, append, attention, 8-bit output
    head, softmax, verification, whose `keep` and token go into the next round. Against the same rounds on the host: lengths,
    tables and tokens equal, and the cache's pages hold what a cache without drafts that failed holds."""
    gen = torch.Generator().manual_seed(11)
    users, heads, kv_heads, dim, page, vocab, drafts = 3, 4, 2, 64, 16, 500, 3
    hidden, per = heads * dim, drafts + 1
    cache = aw.awsrc_kv_cache_alloc(40, kv_heads, dim, page)
    pool = aw.awsrc_kv_pool_alloc(cache, users, 200)
    attn_ws, ws = aw.awsrc_attention_workspace(cache, heads), aw.awsrc_step_workspace()

    def weights(n, k):
        return aw.awsrc_fp8_quantize((torch.randn(n, k, generator=gen) * k ** -0.5).cuda())

    wqkv, wo, head = weights(hidden + 2 * kv_heads * dim, hidden), weights(hidden, hidden), weights(vocab, hidden)
    embed = torch.randn(vocab, hidden, generator=gen).cuda()
    cos, sin = torch.ones(200, dim // 2, device="cuda"), torch.zeros(200, dim // 2, device="cuda")

    def model(ids, batch, n):
        x = embed[ids.long()]
        qkv = aw.awsrc_fp8_linear(x, wqkv, aw.awsrc_fp8_matrix(n, hidden), ws).view(n, heads + 2 * kv_heads, dim)
        q = aw.awsrc_kv_append(cache, batch, qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], cos, sin,
                               attn_ws)
        o = aw.awsrc_paged_attention(cache, batch, q, attn_ws).view(n, hidden)
        x = x + aw.awsrc_fp8_linear(o, wo, aw.awsrc_fp8_matrix(n, hidden), ws)
        return torch.softmax(4 * aw.awsrc_fp8_linear(x, head, aw.awsrc_fp8_matrix(n, hidden), ws), -1)

    # prompts
    lengths = [17, 30, 5]
    n = sum(lengths)
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    start = aw.awsrc_kv_plan(pool, None, cuda_ints(lengths), ws, tok_slot=slots)
    batch = aw.awsrc_kv_batch(start, pool.kv_len, pool.page_table, n, max(lengths), 200)
    prompt = torch.randint(vocab, (n,), generator=gen).to(I32).cuda()
    p = model(prompt, batch, n)
    rows = torch.tensor([sum(lengths[:b + 1]) - 1 for b in range(users)]).cuda()
    _, first = aw.awsrc_verify_drafts(torch.arange(users + 1, dtype=I32, device="cuda"), prompt[rows].contiguous(), p[rows], None,
                                      torch.rand(users, device="cuda"), torch.zeros(users, device="cuda"), ws, max_draft=0)
    assert slots.unique().numel() == n

    # rounds
    ids = torch.zeros(users * per, dtype=I32, device="cuda")
    guess = torch.zeros(users, drafts, dtype=I32, device="cuda")
    u, r = torch.zeros(users * per, device="cuda"), torch.zeros(users, device="cuda")
    keep, add = pool.kv_len.clone(), torch.full((users,), per, dtype=I32, device="cuda")
    q_start = torch.empty(users + 1, dtype=I32, device="cuda")
    pos = torch.empty(users * per, dtype=I32, device="cuda")
    last = first[:, 0].clone()
    accepted, tokens = torch.empty(users, dtype=I32, device="cuda"), torch.empty(users, per, dtype=I32, device="cuda")
    probs = torch.empty(users * per, vocab, device="cuda")
    step = aw.awsrc_kv_batch(q_start, pool.kv_len, pool.page_table, users * per, per, 200)

    def one_round():
        aw.awsrc_kv_plan(pool, keep, add, ws, q_start=q_start, tok_pos=pos)
        ids.view(users, per)[:, 0] = last
        ids.view(users, per)[:, 1:] = guess
        probs.copy_(model(ids, step, users * per))
        aw.awsrc_verify_drafts(q_start, ids, probs, None, u, r, ws, kv_len=pool.kv_len, keep=keep, accepted=accepted, tokens=tokens)
        last.copy_(tokens.gather(1, accepted.long()[:, None])[:, 0])

    state = [t.clone() for t in (pool.page_table, pool.kv_len, pool.free_pages, pool.free_count, keep, last, cache.k.view(torch.uint8),
                                 cache.v.view(torch.uint8), cache.k_exp, cache.v_exp)]

    def restore():
        for t, s in zip((pool.page_table, pool.kv_len, pool.free_pages, pool.free_count, keep, last, cache.k.view(torch.uint8),
                         cache.v.view(torch.uint8), cache.k_exp, cache.v_exp), state):
            t.copy_(s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one_round()  # warm-up; its effects are taken back
        restore()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            one_round()
    torch.cuda.synchronize()

    length = list(lengths)
    rng = random.Random(7)
    total = 0
    for _ in range(12):
        # a guess that is sometimes right: what the model itself put there first, found by running the round greedily
        guess.copy_(torch.randint(vocab, (users, drafts), generator=gen))
        if rng.random() < 0.8:
            saved = [t.clone() for t in (pool.page_table, pool.kv_len, pool.free_pages, pool.free_count, keep, last,
                                         cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_exp, cache.v_exp)]
            for i in range(rng.randrange(1, drafts + 1)):
                graph.replay()
                best = probs.view(users, per, vocab)[:, i].argmax(-1)
                for t, s in zip((pool.page_table, pool.kv_len, pool.free_pages, pool.free_count, keep, last,
                                 cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_exp, cache.v_exp), saved):
                    t.copy_(s)
                guess[:, i] = best.to(I32)
        u.uniform_(0, 0.05)
        r.copy_(torch.rand(users, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.verify(list(range(0, users * per + 1, per)), ids.tolist(), probs.double().tolist(), None, u.tolist(), r.tolist(),
                          drafts, [k + per for k in length])
        assert accepted.tolist() == want[0] and tokens.tolist() == want[1] and keep.tolist() == want[2]
        assert pos.tolist() == [k + i for k in length for i in range(per)]
        assert pool.kv_len.tolist() == [k + per for k in length]
        length = keep.tolist()
        total += sum(want[0])
        held = [row[:-(-(k + per) // page)] for row, k in zip(pool.page_table.tolist(), [v - per for v in pool.kv_len.tolist()])]
        pages = [g for row in held for g in row] + pool.free_pages.tolist()[:pool.free_count.item()]
        assert sorted(pages) == list(range(40))  # every page has one holder
    assert total > 0  # drafts were accepted
    assert aw.awsrc_workspace_status(ws) == 0 and aw.awsrc_workspace_status(attn_ws) == 0
