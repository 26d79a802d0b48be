"""GPU parity of the serving-step calls in forms beside the usual ones: other streams,
launch forms of large vocabularies, thresholds of tiny random numbers, long sums."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def aw():
    import paper_2608_23144_gb300 as aw
    assert torch.cuda.is_available()
    return aw


def cuda_ints(v, dtype=I32):
    return torch.tensor(v, dtype=dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_on_another_stream_than_the_busy_current_one(aw, dtype):
    """A matrix made by the call itself while the current stream has work queued: what the fill would
    overwrite if it came behind that work. The product on the same stream reads the codes."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(300, 1000, generator=gen).to(dtype).cuda()
    want = aw.awsrc_fp8_quantize(x)
    ws = aw.awsrc_step_workspace()
    product = aw.awsrc_fp8_gemm(want, want, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)  # some 10 ms of the current stream
        m = aw.awsrc_fp8_quantize(x, stream=side)
        y = aw.awsrc_fp8_gemm(m, m, ws, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(m.codes.view(torch.uint8), want.codes.view(torch.uint8)) and torch.equal(m.exps, want.exps)
        assert torch.equal(y, product)
    assert aw.awsrc_workspace_status(ws) == 0


def test_older_calls_on_another_stream_than_the_busy_current_one(aw):
    """Backbone, seed search, selection (whose stream starts as zeros) and decoding on a side stream, every
    buffer made by the calls, while the current stream has work queued."""
    from synth import make_module
    m = make_module(256, 512, seed=5, device="cuda")
    prm = aw.params(C=64, P=4, b=4, S=128)

    def run(s=None):
        back = aw.awsrc_rtn_quantize(m["W"], stream=s)
        cands = aw.awsrc_encode_tiles(prm, [m], stream=s)
        out, counts, nbytes = aw.awsrc_select_records(prm, [m], cands, [0.3], stream=s)
        return [back["codes"], back["scales"].view(torch.uint8), cands, counts, nbytes, out, *aw.awsrc_decode_apply(prm, [m], out, -1, stream=s)]

    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(2):
        torch.cuda._sleep(20_000_000)
        got = run(side)
        torch.cuda.synchronize()
        used = int(want[4][0])
        for a, b in zip(got, want):
            assert torch.equal(a[:used] if b is want[5] else a, b[:used] if b is want[5] else b)
    torch.cuda._sleep(20_000_000)
    assert aw.awsrc_verify_reciprocal(0x3F800000, 0x3F900000, stream=side) == 0


def test_verify_thresholds_of_tiny_random_numbers(aw):
    """r C_V just above a whole number of units with r below 2^-40: weights k, rest, of T = ceil(k 2^65 / m) units in all, and
    r = m 2^-65, so k <= r T < k + 2^-18: the first weight does not reach above it, the second does. m is odd, so r has bits
    below 2^-64. Random numbers down to the smallest of binary32 beside them."""
    from test_gpu_step import check
    rows, r = [], []
    for m in (2 ** 23 + 1, 2 ** 23 + 4097, 2 ** 24 - 1, 12345679):
        for k in (1, 3, 7):
            total = -(-k * 2 ** 65 // m)
            assert total < 2 ** 45 and k * 2 ** 65 <= m * total < k * 2 ** 65 + m
            rest = total - k
            rows.append([k, rest >> 23 << 23, rest & (2 ** 23 - 1), 0, 0])
            r.append(m * 2.0 ** -65)
    for tiny in (2.0 ** -149, 2.0 ** -127, 2.0 ** -64, 2.0 ** -46, 3 * 2.0 ** -47, 2.0 ** -45, 1 - 2.0 ** -24):
        rows.append([1, 2, 2 ** 44, 0, 1])
        r.append(tiny)
    p = (torch.tensor(rows, dtype=torch.float64) * 2.0 ** -45).float()
    assert torch.equal(p.double() * 2.0 ** 45, torch.tensor(rows, dtype=torch.float64))
    n = len(rows)
    for q in (None, torch.zeros_like(p)):
        want = check(aw, list(range(n + 1)), [0] * n, p, q, torch.rand(n), torch.tensor(r, dtype=F32), 0, [5] * n)
        assert [t[0] for t in want[1][:12]] == [1] * 12


@pytest.mark.parametrize("bad,value", [(1, -1), (20, 50), (33, 2 ** 31 - 1), (36, -5), (65, 50), (70, 99)])
@pytest.mark.parametrize("stop", [0, 31, 32, 40, 70])
def test_verify_reports_drafts_outside_wherever_they_are(aw, bad, value, stop):
    """70 drafts, the one at `stop` refused, the one at `bad` (counted from 1) outside the vocabulary: reported, whether it is
    looked at for acceptance or not, and never accepted."""
    from test_gpu_step import check
    gen = torch.Generator().manual_seed(bad)
    p = torch.softmax(torch.randn(71, 50, generator=gen) * 3, -1)
    ids = [0] + p[:-1].argmax(-1).tolist()
    ids[bad] = value
    u = torch.zeros(71)
    u[stop:] = 1.0
    want = check(aw, [0, 71], ids, p, None, u, torch.rand(1, generator=gen), 70, [500], flags=8)
    assert want[0] == [min(stop, bad - 1)]


def test_a_captured_round_with_a_pool_that_runs_out(aw):
    """Five users, rounds of drafts as one captured graph, pages for about half of what they want. A user that finds no room has no
    rows in the round; it goes on with the token it had (verification gives -1 for it) once others' pages come back. Rows of
    the round are found through the maps, so that they are right whoever was admitted. Every round against the definitions."""
    import step_ref as ref
    gen = torch.Generator().manual_seed(21)
    users, heads, kv_heads, dim, page, vocab, drafts, pages = 5, 4, 2, 64, 16, 300, 3, 7
    hidden, per, most = heads * dim, drafts + 1, 128
    cache = aw.awsrc_kv_cache_alloc(pages, kv_heads, dim, page)
    pool = aw.awsrc_kv_pool_alloc(cache, users, most)
    attn_ws, ws, n_tok = aw.awsrc_attention_workspace(cache, heads), aw.awsrc_step_workspace(), users * per

    def weights(n, k):
        return aw.awsrc_fp8_quantize((torch.randn(n, k, generator=gen) * k ** -0.5).cuda())

    wqkv, wo, head = weights(hidden + 2 * kv_heads * dim, hidden), weights(hidden, hidden), weights(vocab, hidden)
    embed = torch.randn(vocab, hidden, generator=gen).cuda()
    x8 = aw.awsrc_fp8_matrix(n_tok, hidden)
    q_start, keep = torch.empty(users + 1, dtype=I32, device="cuda"), torch.zeros(users, dtype=I32, device="cuda")
    seq, pos = (torch.empty(n_tok, dtype=I32, device="cuda") for _ in range(2))
    add, last = torch.full((users,), per, dtype=I32, device="cuda"), cuda_ints([3, 1, 4, 1, 5])
    guess = torch.zeros(users, drafts, dtype=I32, device="cuda")
    u, r = torch.zeros(n_tok, device="cuda"), torch.zeros(users, device="cuda")
    ids, probs = torch.zeros(n_tok, dtype=I32, device="cuda"), torch.zeros(n_tok, vocab, device="cuda")
    accepted, tokens = torch.empty(users, dtype=I32, device="cuda"), torch.empty(users, per, dtype=I32, device="cuda")
    step = aw.awsrc_kv_batch(q_start, pool.kv_len, pool.page_table, n_tok, per, most)

    def one_round():
        aw.awsrc_kv_plan(pool, keep, add, ws, q_start=q_start, tok_seq=seq, tok_pos=pos)
        who = seq.long().clamp(min=0)
        window = torch.cat([last[:, None], guess], 1)
        ids.copy_(window[who, (pos - keep[who]).long().clamp(0, drafts)])
        x = embed[ids.long()]
        qkv = aw.awsrc_fp8_linear(x, wqkv, x8, ws).view(n_tok, -1, dim)
        q = aw.awsrc_kv_append(cache, step, qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], None, None,
                               attn_ws, q_out=torch.zeros(n_tok, heads, dim, device="cuda"))
        o = aw.awsrc_paged_attention(cache, step, q, attn_ws, out=torch.zeros(n_tok, heads, dim, device="cuda")).view(n_tok, hidden)
        x = x + aw.awsrc_fp8_linear(o, wo, x8, ws)
        probs.copy_(torch.softmax(4 * aw.awsrc_fp8_linear(x, head, x8, ws), -1))
        aw.awsrc_verify_drafts(q_start, ids, probs, None, u, r, ws, kv_len=pool.kv_len, keep=keep, accepted=accepted, tokens=tokens)
        token = tokens.gather(1, accepted.long()[:, None])[:, 0]
        last.copy_(torch.where(q_start[1:] > q_start[:-1], token, last))  # who had no rows keeps its token

    state = (pool.page_table, pool.kv_len, pool.free_pages, pool.free_count, keep, last)
    before = [s.clone() for s in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one_round()
        for s, b in zip(state, before):
            s.copy_(b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            one_round()
    torch.cuda.synchronize()

    table, length, free, count = [pool.page_table.tolist(), [0] * users, pool.free_pages.tolist(), pages]
    kept, mine, waited, resumed = [0] * users, last.tolist(), set(), set()
    for i in range(30):
        adds = [per if k + per <= most else 0 for k in kept]
        if i % 6 == 5:  # the longest ends: its pages come back, a new text of its begins
            b = max(range(users), key=lambda b: kept[b])
            kept[b], mine[b] = 0, 7
            keep[b], last[b] = 0, 7
        add.copy_(torch.tensor(adds, dtype=I32))
        guess.copy_(torch.randint(vocab, (users, drafts), generator=gen))
        u.uniform_(0, 0.02)
        r.copy_(torch.rand(users, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        table, length, free, count, starts, seqs, poss, _, flags = ref.plan(page, table, length, free, count, kept, adds, n_tok)
        assert aw.awsrc_workspace_status(ws) == flags and aw.awsrc_workspace_status(attn_ws) == 0
        assert q_start.tolist() == starts and seq.tolist() == seqs and pos.tolist() == poss
        assert pool.kv_len.tolist() == length and pool.page_table.tolist() == table and pool.free_count.item() == count
        fed, g = ids.tolist(), guess.tolist()
        for b in range(users):
            rows = fed[starts[b]:starts[b + 1]]
            assert rows == ([mine[b]] + g[b])[:len(rows)]
            if rows and b in waited:
                resumed.add(b)
            if adds[b] and not rows:
                waited.add(b)
        want = ref.verify(starts, fed, probs.double().tolist(), None, u.tolist(), r.tolist(), drafts, length)
        assert accepted.tolist() == want[0] and tokens.tolist() == want[1] and keep.tolist() == want[2]
        kept = want[2]
        mine = [want[1][b][want[0][b]] if starts[b + 1] > starts[b] else mine[b] for b in range(users)]
        assert last.tolist() == mine and min(mine) >= 0
    assert waited and resumed  # some had to wait, and went on


@pytest.mark.parametrize("p_dtype,q_dtype", [(F32, BF16), (BF16, F32), (F32, F32), (BF16, BF16), (F32, None)])
@pytest.mark.parametrize("vocab,n_seq", [(131071, 2), (131072, 1), (151936, 1), (151937, 19), (2 ** 18 - 1, 3), (2 ** 18, 1)])
def test_verify_large_vocabularies(aw, p_dtype, q_dtype, vocab, n_seq):
    """1024 threads (131072 columns and up to 19 sequences) and what is beside them, up to the largest vocabulary; a model's and a
    draft model's probabilities of the same type and of two; thresholds in every part of a row."""
    from test_gpu_step import check
    gen = torch.Generator().manual_seed(vocab + n_seq)
    n = 2 * n_seq if n_seq < 4 else n_seq + 1  # one draft each, or one for the last sequence alone
    starts = list(range(0, n + 1, 2)) if n_seq < 4 else list(range(n_seq)) + [n]
    x = torch.randn(n, vocab, generator=gen)
    p = torch.softmax(x, -1).to(p_dtype)
    q = None if q_dtype is None else torch.softmax(x + torch.randn(n, vocab, generator=gen), -1).to(q_dtype)
    ids = torch.randint(vocab, (n,), generator=gen).tolist()
    ids[-1] = vocab - 1
    r = (torch.arange(n_seq) + torch.rand(n_seq, generator=gen)) / n_seq
    want = check(aw, starts, ids, p, q, torch.rand(n, generator=gen), r, 1, [100] * n_seq, pad=vocab % 4)
    assert all(-1 not in t[:a + 1] for a, t in zip(*want[:2]))


@pytest.mark.parametrize("p_dtype,q_dtype", [(F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("vocab,pad", [(1, 0), (31, 1), (1000, 0), (1000, 4), (1001, 3), (4099, 0)])
def test_verify_probabilities_of_two_types(aw, p_dtype, q_dtype, vocab, pad):
    """Rows that start on each type's vector boundary, on one of them, and on neither."""
    from test_gpu_step import check, rows_of
    rng, gen = random.Random(vocab + pad), torch.Generator().manual_seed(vocab + pad)
    lens = [1, 4, 0, 7, 2, 3]
    starts = [sum(lens[:b]) for b in range(len(lens) + 1)]
    n = starts[-1]
    p, q = rows_of(rng, gen, n, vocab, "wide", torch.float64)
    p, q = p.to(p_dtype), q.to(q_dtype)
    ids = [rng.randrange(vocab) for _ in range(n)]
    for t in range(n - 1):
        if rng.random() < 0.6:
            ids[t + 1] = int(p[t].argmax())
    check(aw, starts, ids, p, q, torch.rand(n, generator=gen), torch.rand(len(lens), generator=gen), 6,
          [rng.randrange(20, 900) for _ in lens], pad=pad)


@pytest.mark.parametrize("n_seq", [1, 20, 700])
def test_verify_the_largest_sums(aw, n_seq):
    """Every entry of the largest vocabulary 1 (or above): running sums up to 2^63 units. The token is floor(r 2^18)."""
    vocab = 2 ** 18
    p = torch.ones(n_seq, vocab, device="cuda", dtype=BF16)
    p[:, ::3] = 7.0
    r = torch.rand(n_seq, generator=torch.Generator().manual_seed(n_seq))
    r[0] = 1 - 2.0 ** -24
    ws = aw.awsrc_step_workspace()
    starts = torch.arange(n_seq + 1, dtype=I32).cuda()
    ids = torch.zeros(n_seq, dtype=I32, device="cuda")
    acc, tok = aw.awsrc_verify_drafts(starts, ids, p, None, torch.zeros(n_seq, device="cuda"), r.cuda(), ws, max_draft=0)
    assert tok[:, 0].tolist() == (r.double() * vocab).floor().int().tolist() and not acc.any()
    assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("n_seq", [2048, 2049, 8192])
def test_plan_of_the_most_sequences(aw, n_seq):
    """Around the change to larger thread blocks, and as many sequences as there may be: decoding with pages for all, drafts
    that go back, prompts that do not all fit."""
    from test_gpu_step import Pool
    rng = random.Random(n_seq)
    lengths = [rng.choice([0, 1, 15, 16, 17, rng.randrange(90)]) for _ in range(n_seq)]
    pool = Pool(aw, rng, n_seq, 16, 14, lengths, spare=n_seq // 2)
    flags = [pool.step(None, [1] * n_seq, n_seq)]
    keep = [max(0, k - rng.randrange(4)) for k in pool.length]
    flags.append(pool.step(keep, [rng.randrange(5) for _ in keep], 5 * n_seq))
    keep = [0 if rng.random() < 0.1 else k for k in pool.length]
    flags.append(pool.step(keep, [rng.randrange(90) if k == 0 else 1 for k in keep], 3 * n_seq))
    assert flags[0] in (0, 16) and 16 in flags
    assert pool.step([0] * n_seq, [0] * n_seq, 3) == 0
