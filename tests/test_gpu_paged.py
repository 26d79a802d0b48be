"""GPU parity of the paged 8-bit cache: awsrc_kv_append bit for bit with the
header's recipe, awsrc_paged_attention within derived bounds of the definition in
64 bits (tests/paged_ref.py)."""
import math

import pytest
import torch

import paged_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def aw():
    import paper_2608_23144_gb300 as aw
    assert torch.cuda.is_available()
    return aw


def make_batch(aw, gen, new, kv, page, spare=2, slack=0):
    """(batch handle, page table on the host, pages of the cache): pages in random order, unused entries -1."""
    used = [-(-(k + slack) // page) for k in kv]
    pages = sum(used) + spare
    order = torch.randperm(pages, generator=gen)
    table = torch.full((len(kv), max(used + [1])), -1, dtype=torch.int32)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at:at + u].int()
        at += u
    return step_batch(aw, new, kv, table), table, pages


def step_batch(aw, new, kv, table):
    q_start = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32)
    return aw.awsrc_kv_batch(q_start.cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), table.cuda(), sum(new),
                             max(new), max(kv))


def tables(n, half, gen):
    ang = torch.rand(n, half, generator=gen, dtype=torch.float64) * 6.3
    return ang.cos().float(), ang.sin().float()


def random_cache(aw, gen, pages, heads, dim, page):
    """A cache with every block filled; scales over a range of exponents."""
    c = aw.awsrc_kv_cache_alloc(pages, heads, dim, page)
    for codes, exps in ((c.k, c.k_exp), (c.v, c.v_exp)):
        x = torch.randn(codes.shape, generator=gen) * 120
        codes.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn))
        exps.copy_(torch.randint(-10, -4, exps.shape, generator=gen).to(torch.int8))
    return c


def assert_cache_equal(got, want):
    for w in "kv":
        assert torch.equal(got.exp[w], want.exp[w]), w
        assert torch.equal(got.code[w], want.code[w]), w


# ------------------------------------------------------------------- append

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,dim,page,rotary,inter", [
    (16, 2, 128, 64, 128, False), (7, 1, 128, 16, 128, True), (12, 12, 64, 32, 32, True), (4, 2, 64, 128, 32, False),
    (6, 3, 64, 16, 20, False), (2, 1, 128, 128, 0, False)])
def test_append_follows_the_recipe(aw, dtype, heads, kv_heads, dim, page, rotary, inter):
    """Prompts, a chunk that starts inside a page, single tokens whose size grows and shrinks: every code, exponent
    and rotated query of every step, sequences of no new tokens among them; q, k, v as slices of one row tensor."""
    gen = torch.Generator().manual_seed(heads * 1000 + page)
    steps = [([page + 3, 1, 0, 2 * page], 1.0), ([5, page - 1, 1, 0], 3.0), ([1, 1, 1, 1], 40.0), ([1, 1, 1, 1], 0.01),
             ([0, 2, 1, 1], 300.0)]
    kv_end = [sum(s[0][b] for s in steps) for b in range(4)]
    _, table, pages = make_batch(aw, gen, steps[0][0], kv_end, page)
    cache = random_cache(aw, gen, pages, kv_heads, dim, page)
    want = ref.Cache.of(cache)
    ws = aw.awsrc_attention_workspace(cache, heads)
    cos, sin = tables(max(kv_end), rotary // 2, gen) if rotary else (None, None)
    dcos, dsin = (cos.cuda(), sin.cuda()) if rotary else (None, None)
    kv = [0] * 4
    for new, size in steps:
        kv = [a + b for a, b in zip(kv, new)]
        qkv = (torch.randn(sum(new), heads + 2 * kv_heads, dim, generator=gen) * size).to(dtype)
        qkv[:, heads:heads + kv_heads, 0] *= 7
        d = qkv.cuda()
        cut = (slice(0, heads), slice(heads, heads + kv_heads), slice(heads + kv_heads, None))
        got_q = aw.awsrc_kv_append(cache, step_batch(aw, new, kv, table), *(d[:, c] for c in cut), dcos, dsin, ws,
                                   interleaved=inter)
        want_q = ref.append(want, *(qkv[:, c] for c in cut), new, kv, table, cos, sin, inter)
        assert torch.equal(got_q.cpu(), want_q.to(dtype))
        assert_cache_equal(ref.Cache.of(cache), want)
    assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_values_are_within_half_a_code_of_64_bits(aw, dtype):
    """The cached values against the 64-bit rotation: half an e4m3 step (2^-4 of the value, 2^-10 of the scale below
    the normal range), the rotation's three binary32 roundings (each at most 2^-24 of |x1| + |x2|), and what a later
    growth of the scale rounds away (2^-10 of the final scale)."""
    gen = torch.Generator().manual_seed(3)
    new, heads, page = [150, 33], 2, 64
    batch, table, pages = make_batch(aw, gen, new, new, page)
    cache = aw.awsrc_kv_cache_alloc(pages, heads, 128, page)
    x = (torch.randn(3, sum(new), heads, 128, generator=gen) * torch.exp(torch.randn(128, generator=gen))).to(dtype)
    cos, sin = tables(200, 64, gen)
    aw.awsrc_kv_append(cache, batch, *x.cuda(), cos.cuda(), sin.cuda(), aw.awsrc_attention_workspace(cache, heads))
    c = ref.Cache.of(cache)
    at = 0
    for b, n in enumerate(new):
        pages_b = [int(p) for p in table[b][:-(-n // page)]]
        for h in range(heads):
            k, v = x[1, at:at + n, h].double(), x[2, at:at + n, h].double()
            a, z = k[:, :64], k[:, 64:]
            co, si = cos[:n].double(), sin[:n].double()
            turned = torch.cat((a * co - z * si, z * co + a * si), 1)
            reach = (a.abs() + z.abs()).repeat(1, 2)
            for which, want, slack in (("k", turned, 3 * 2.0 ** -24 * reach), ("v", v, 0.0)):
                scale = torch.exp2(c.exp[which][pages_b, h].double()).repeat_interleave(page)[:n, None]
                err = (c.values(which, pages_b, h, n) - want).abs()
                assert (err <= torch.maximum(want.abs() * 2.0 ** -4, scale * 2.0 ** -10) + 1.1 * slack).all()
        at += n


@pytest.mark.parametrize("off", [1, 4])
def test_append_takes_any_strides_and_alignment(aw, off):
    """Rows that are not 16-byte aligned (element by element) give what aligned rows give, in place too."""
    gen = torch.Generator().manual_seed(4)
    new, kv = [70, 3], [70, 103]
    batch, table, pages = make_batch(aw, gen, new, kv, 32)
    x = torch.randn(3, 73, 4, 64, generator=gen).to(BF16).cuda()
    cos, sin = (t.cuda() for t in tables(103, 32, gen))
    a, b = (aw.awsrc_kv_cache_alloc(pages, 4, 64, 32) for _ in range(2))
    ws = aw.awsrc_attention_workspace(a, 4)
    want = aw.awsrc_kv_append(a, batch, *x, cos, sin, ws)
    wide = torch.zeros(3, 4, 73, 64 + off, dtype=BF16, device="cuda")  # heads outermost, rows at odd addresses
    wide[..., off:] = x.transpose(1, 2)
    y = wide[..., off:].transpose(1, 2)
    got = aw.awsrc_kv_append(b, batch, *y, cos, sin, ws, q_out=y[0])
    assert got.data_ptr() == y[0].data_ptr() and torch.equal(got, want)
    assert torch.equal(a.k.view(torch.uint8), b.k.view(torch.uint8))
    assert torch.equal(a.v.view(torch.uint8), b.v.view(torch.uint8))
    assert torch.equal(a.k_exp, b.k_exp) and torch.equal(a.v_exp, b.v_exp)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 1e13])
def test_append_marks_blocks_that_cannot_be_scaled(aw, value):
    """A non-finite (or too large) element marks its block alone, keeps it marked, and a page written from row 0 again
    is clean; attention over a marked block gives NaN for the kv head that reads it and no other."""
    gen = torch.Generator().manual_seed(5)
    _, table, pages = make_batch(aw, gen, [20], [40], 16)
    cache = aw.awsrc_kv_cache_alloc(pages, 2, 64, 16)
    ws = aw.awsrc_attention_workspace(cache, 2)
    want = ref.Cache.of(cache)
    kv = 0
    for n, bad in ((20, None), (1, "v"), (2, None), (17, "k")):
        kv += n
        q, k, v = torch.randn(3, n, 2, 64, generator=gen)
        if bad:
            (k if bad == "k" else v)[0, 1, 5] = value
        batch = step_batch(aw, [n], [kv], table)
        aw.awsrc_kv_append(cache, batch, q.cuda(), k.cuda(), v.cuda(), None, None, ws)
        ref.append(want, q, k, v, [n], [kv], table, None, None, False)
        assert_cache_equal(ref.Cache.of(cache), want)
    assert (want.exp["v"] == ref.E_NAN).any() and (want.exp["k"] == ref.E_NAN).any()
    lse = torch.empty(1, 2, device="cuda")
    out = aw.awsrc_paged_attention(cache, step_batch(aw, [1], [kv], table), q[:1].cuda(), ws, lse=lse)
    assert torch.isnan(out[0, 1]).all() and torch.isfinite(out[0, 0]).all()
    batch = step_batch(aw, [40], [40], table)  # the pages' next sequence
    x = torch.randn(3, 40, 2, 64, generator=gen)
    aw.awsrc_kv_append(cache, batch, *x.cuda(), None, None, ws)
    ref.append(want, *x, [40], [40], table, None, None, False)
    assert_cache_equal(ref.Cache.of(cache), want)
    assert not (want.exp["v"][table[0].long()] == ref.E_NAN).any()
    assert torch.isfinite(aw.awsrc_paged_attention(cache, batch, x[0].cuda(), ws)).all()


def test_entries_that_cannot_be_right_are_skipped_and_reported(aw):
    """Pages outside the cache, more new tokens than tokens, lengths beyond the table, starts out of order, positions
    beyond the rotation tables: bit 3, and the other sequences as if they were alone."""
    gen = torch.Generator().manual_seed(6)
    new, kv = [4, 4, 4], [36, 40, 20]
    _, table, pages = make_batch(aw, gen, new, kv, 16)
    x = torch.randn(3, 12, 2, 64, generator=gen).cuda()
    cos, sin = (t.cuda() for t in tables(64, 32, gen))
    base = random_cache(aw, gen, pages, 2, 64, 16)
    start = [0, 4, 8, 12]

    def run(t, s, k, rows=64):
        c = aw.awsrc_kv_cache(*(b.clone() for b in (base.k, base.v, base.k_exp, base.v_exp)))
        ws = aw.awsrc_attention_workspace(c, 2)
        batch = aw.awsrc_kv_batch(torch.tensor(s, dtype=torch.int32).cuda(), torch.tensor(k, dtype=torch.int32).cuda(),
                                  t.cuda(), 12, 4, 40)
        q = aw.awsrc_kv_append(c, batch, *x, cos[:rows], sin[:rows], ws, q_out=torch.zeros_like(x[0]))
        f1 = aw.awsrc_workspace_status(ws)
        out = aw.awsrc_paged_attention(c, batch, x[0], ws, out=torch.zeros_like(x[0]))
        return c, q, out, f1, aw.awsrc_workspace_status(ws)

    good, q0, out0, f1, f2 = run(table, start, kv)
    assert f1 == 0 and f2 == 0
    t2 = table.clone()
    t2[1, 2] = pages + 7  # the page that sequence 1's new tokens go to
    t3 = table.clone()
    t3[1, 2] = -5
    cases = [(t2, start, kv, 64, True), (t3, start, kv, 64, True), (table, start, [36, 3, 20], 64, True),
             (table, start, [36, 16 * table.shape[1] + 1, 20], 64, True), (table, start, [36, -1, 20], 64, True),
             (table, [0, 4, 8, 13], kv, 64, False), (table, start, kv, 38, None)]
    for t, s, k, rows, middle in cases:
        c, q, out, f1, f2 = run(t, s, k, rows)
        assert f1 == 8 and f2 == (8 if middle is not None else 0)
        keep = slice(0, 4) if middle is False else [0, 1, 2, 3, 8, 9, 10, 11]
        assert torch.equal(q[keep], q0[keep]) and torch.equal(out[keep], out0[keep])
        for b in (0, 2) if middle is not False else (0,):
            pg = table[b][table[b] >= 0].long().cuda()
            for have, should in ((c.k, good.k), (c.v, good.v)):
                assert torch.equal(have.view(torch.uint8)[pg], should.view(torch.uint8)[pg])


# ---------------------------------------------------------------- attention

def check_attention(aw, cache, q, new, kv, table, causal, scale=None, batch=None, ws=None, strided=False):
    n, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    c = ref.Cache.of(cache)
    ws = aw.awsrc_attention_workspace(cache, heads) if ws is None else ws
    dq = q.cuda()
    out = torch.full((n, heads, dim), 7.0, dtype=q.dtype, device="cuda")
    if strided:
        dq = torch.zeros(heads, n, dim + 3, dtype=q.dtype, device="cuda")[..., 3:].transpose(0, 1).copy_(dq)
        out = torch.full((n, heads + 1, dim + 1), 7.0, dtype=q.dtype, device="cuda")[:, 1:, 1:]
    lse = torch.full((n, heads), 7.0, device="cuda")
    batch = step_batch(aw, new, kv, table) if batch is None else batch
    aw.awsrc_paged_attention(cache, batch, dq, ws, sm_scale=scale, causal=causal, out=out, lse=lse)
    assert aw.awsrc_workspace_status(ws) == 0
    eps = (2.0 ** -22, 2.0 ** -22) if q.dtype == F32 else (0.0, 2.0 ** -9)
    want, wl, ob, lb = ref.attention(c, q, new, kv, table, scale, causal, *eps)
    got = out.cpu().double()
    if q.dtype == BF16:
        ob = ob + (want.abs() + ob) * 2.0 ** -9  # out is rounded once
    empty = torch.isinf(wl)
    assert torch.equal(torch.isinf(lse.cpu()), empty) and (got[empty] == 0).all()
    assert ((got - want).abs() <= ob + 1e-30).all(), float(((got - want).abs() - ob).max())
    assert ((lse.cpu().double() - wl).abs()[~empty] <= lb[~empty]).all()
    return out


LAYOUTS = [(16, 2, 128), (7, 1, 128), (10, 2, 128), (3, 3, 64), (14, 1, 64), (48, 2, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,dim", LAYOUTS)
@pytest.mark.parametrize("page", [16, 64, 128])
def test_decode_steps(aw, dtype, heads, kv_heads, dim, page):
    """One new token per sequence, lengths around every block edge, an empty sequence and one without a query."""
    gen = torch.Generator().manual_seed(heads + page)
    kv = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 0, 9, 1111]
    new = [1] * len(kv)
    new[12] = new[13] = 0
    _, table, pages = make_batch(aw, gen, new, kv, page)
    cache = random_cache(aw, gen, pages, kv_heads, dim, page)
    check_attention(aw, cache, torch.randn(sum(new), heads, dim, generator=gen).to(dtype), new, kv, table, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(16, 2, 128, 64), (7, 1, 128, 16), (3, 3, 64, 32), (40, 8, 128, 128),
                                                     (14, 2, 64, 16)])
def test_ragged_queries(aw, dtype, causal, heads, kv_heads, dim, page):
    """Drafts, chunks and prompts of every kind in one batch, single tokens beside them."""
    gen = torch.Generator().manual_seed(page + heads)
    new = [1, 5, 64, 0, 130, 1, 33, 17, 200]
    kv = [700, 5, 64, 40, 300, 1, 1000, 90, 200]
    _, table, pages = make_batch(aw, gen, new, kv, page)
    cache = random_cache(aw, gen, pages, kv_heads, dim, page)
    q = torch.randn(sum(new), heads, dim, generator=gen).to(dtype)
    check_attention(aw, cache, q, new, kv, table, causal, strided=not causal)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,kv", [([1], [40000]), ([3], [9001]), ([1, 1], [1, 30000]), ([300], [5000]), ([1000], [1000])])
def test_long_sequences_are_joined(aw, dtype, new, kv):
    """Few rows over a long axis: many blocks share a tile; repeated calls give the same bits."""
    gen = torch.Generator().manual_seed(kv[0])
    _, table, pages = make_batch(aw, gen, new, kv, 64)
    cache = random_cache(aw, gen, pages, 1, 128, 64)
    q = (torch.randn(sum(new), 5, 128, generator=gen) * 0.3).to(dtype)
    ws = aw.awsrc_attention_workspace(cache, 5)
    a = check_attention(aw, cache, q, new, kv, table, True, ws=ws)
    for _ in range(3):
        assert torch.equal(check_attention(aw, cache, q, new, kv, table, True, ws=ws), a)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
def test_scales_and_scores_of_every_size(aw, dtype, new):
    """Blocks whose scales differ by 2^60, scores far apart, query rows of all sizes, rows of zeros."""
    gen = torch.Generator().manual_seed(8)
    kv = [300]
    _, table, pages = make_batch(aw, gen, [new], kv, 16)
    cache = random_cache(aw, gen, pages, 2, 64, 16)
    cache.v_exp.copy_(torch.randint(-32, 31, cache.v_exp.shape, generator=gen).to(torch.int8))
    cache.k_exp.copy_(torch.randint(-14, -5, cache.k_exp.shape, generator=gen).to(torch.int8))
    q = torch.randn(new, 6, 64, generator=gen) * 10.0 ** torch.arange(-4.0, 2.0)[None, :, None]
    q[:, 3] = 0
    check_attention(aw, cache, q.to(dtype), [new], kv, table, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 70])
def test_bytes_past_the_end_do_not_matter(aw, dtype, new):
    """Rows of the last page that hold no token, pages of no sequence and table entries past the end: NaN codes, marked
    exponents, page numbers out of range."""
    gen = torch.Generator().manual_seed(9)
    for kv in ([new + 1], [new + 13], [new + 63]):
        _, table, pages = make_batch(aw, gen, [new], kv, 64, slack=64)
        cache = random_cache(aw, gen, pages, 1, 128, 64)
        q = torch.randn(new, 4, 128, generator=gen).to(dtype)
        a = check_attention(aw, cache, q, [new], kv, table, True)
        used = table[0][:-(-kv[0] // 64)].long()
        idle = [p for p in range(pages) if p not in used.tolist()]
        for codes, exps in ((cache.k, cache.k_exp), (cache.v, cache.v_exp)):
            codes.view(torch.uint8)[idle] = 0x7F
            exps[idle] = -128
        r = (kv[0] - 1) % 64 + 1  # rows of the last page in use
        cache.k.view(torch.uint8)[used[-1], :, :, r:] = 0xFF
        t = torch.arange(64).view(4, 1, 16).expand(4, 128, 16) >= r
        raw = cache.v.view(torch.uint8)
        raw[used[-1], 0] = torch.where(t.cuda(), 0x7F, raw[used[-1], 0])
        table[0, len(used):] = 10 ** 6
        batch = step_batch(aw, [new], kv, table)
        out = aw.awsrc_paged_attention(cache, batch, q.cuda(), aw.awsrc_attention_workspace(cache, 4))
        assert torch.equal(out, a)


def test_caches_beyond_32_bit_offsets(aw):
    """Pages whose bytes lie past 4 GiB: appended and read like any others."""
    gen = torch.Generator().manual_seed(10)
    page, heads = 128, 8
    pages = (1 << 32) // (page * heads * 128) + 40
    cache = aw.awsrc_kv_cache_alloc(pages, heads, 128, page)
    far = pages - 3
    table = torch.tensor([[far, 1, far + 2]], dtype=torch.int32)
    x = torch.randn(3, 300, heads, 128, generator=gen)
    batch = step_batch(aw, [300], [300], table)
    ws = aw.awsrc_attention_workspace(cache, heads)
    q = aw.awsrc_kv_append(cache, batch, *x.cuda(), None, None, ws)
    small = aw.awsrc_kv_cache_alloc(3, heads, 128, page)
    b2 = step_batch(aw, [300], [300], torch.tensor([[0, 1, 2]], dtype=torch.int32))
    aw.awsrc_kv_append(small, b2, *x.cuda(), None, None, ws)
    pg = table[0].long().cuda()
    assert torch.equal(cache.k.view(torch.uint8)[pg], small.k.view(torch.uint8))
    assert torch.equal(cache.v.view(torch.uint8)[pg], small.v.view(torch.uint8))
    for dt in (BF16, F32):
        for qq, a, b in ((q, batch, b2), (q[-1:].contiguous(), step_batch(aw, [1], [300], table),
                                          step_batch(aw, [1], [300], torch.tensor([[0, 1, 2]], dtype=torch.int32)))):
            qq = qq.to(dt)
            assert torch.equal(aw.awsrc_paged_attention(cache, a, qq, ws), aw.awsrc_paged_attention(small, b, qq, ws))
    assert aw.awsrc_workspace_status(ws) == 0


def test_lengths_are_read_when_the_kernels_run(aw):
    """A captured step follows the lengths in the batch's arrays; another stream works like the default one."""
    gen = torch.Generator().manual_seed(11)
    kv = [100, 37]
    _, table, pages = make_batch(aw, gen, [1, 1], [130, 60], 16)
    batch = step_batch(aw, [1, 1], kv, table)
    base = random_cache(aw, gen, pages, 2, 64, 16)
    caches = [aw.awsrc_kv_cache(*(b.clone() for b in (base.k, base.v, base.k_exp, base.v_exp))) for _ in range(2)]
    cos, sin = (t.cuda() for t in tables(200, 32, gen))
    xs = torch.randn(12, 3, 2, 2, 64, generator=gen).cuda()
    x = xs[0].clone()
    out, q = torch.empty_like(x[0]), torch.empty_like(x[0])
    ws = [aw.awsrc_attention_workspace(c, 2) for c in caches]

    def step(c, w, b, t):
        aw.awsrc_kv_append(c, b, *t, cos, sin, w, q_out=q)
        aw.awsrc_paged_attention(c, b, q, w, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(caches[0], ws[0], batch, x)
    torch.cuda.synchronize()
    for i in range(12):
        x.copy_(xs[i])
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        step(caches[1], ws[1], step_batch(aw, [1, 1], [k + i for k in kv], table), xs[i])
        torch.cuda.synchronize()
        assert torch.equal(out, first), i
        batch.kv_len += 1
    assert torch.equal(caches[0].k.view(torch.uint8), caches[1].k.view(torch.uint8))


def test_empty_batches_do_nothing(aw):
    cache = aw.awsrc_kv_cache_alloc(2, 1, 64, 16)
    ws = aw.awsrc_attention_workspace(cache, 2)
    table = torch.zeros(1, 1, dtype=torch.int32)
    n0 = aw.awsrc_kernel_launches()
    b = step_batch(aw, [0], [5], table)
    q, k = torch.empty(0, 2, 64, device="cuda"), torch.empty(0, 1, 64, device="cuda")
    assert aw.awsrc_kv_append(cache, b, q, k, k, None, None, ws).shape == (0, 2, 64)
    assert aw.awsrc_paged_attention(cache, b, q, ws).shape == (0, 2, 64)
    assert aw.awsrc_kernel_launches() == n0 and aw.awsrc_workspace_status(ws) == 0


def test_waits_that_run_out_are_reported(aw):
    """The tensor-memory kernel's bounded waits: its copies stop after some blocks (100 ms limit), the call returns, the
    fault word says so and the next call works on a workspace made ready again."""
    gen = torch.Generator().manual_seed(12)
    new, kv = [300, 40], [9000, 400]  # shares of 4 blocks and more
    _, table, pages = make_batch(aw, gen, new, kv, 32)
    cache = random_cache(aw, gen, pages, 2, 128, 32)
    q = torch.randn(sum(new), 6, 128, generator=gen).to(BF16)
    for stall in (0, 1, 3):
        ws = aw.awsrc_attention_workspace(cache, 6)
        aw.awsrc_set_wait_test(100_000_000, stall)
        try:
            aw.awsrc_paged_attention(cache, step_batch(aw, new, kv, table), q.cuda(), ws)
            assert aw.awsrc_workspace_status(ws) == 4
        finally:
            aw.awsrc_set_wait_test()
    check_attention(aw, cache, q, new, kv, table, True)


@pytest.mark.parametrize("dtype,new", [(F32, 1), (F32, 40), (BF16, 2)])
def test_waits_of_the_row_kernel_that_run_out_are_reported(aw, dtype, new):
    """The same for the kernel of few rows, whose rings take blocks of 64 tokens: one ring of a thread block's share, or
    four. 70000 tokens of two heads over at most 304 blocks give each ring two blocks and more."""
    gen = torch.Generator().manual_seed(13)
    _, table, pages = make_batch(aw, gen, [new], [70000], 64)
    cache = random_cache(aw, gen, pages, 2, 128, 64)
    q = torch.randn(new, 6, 128, generator=gen).to(dtype)
    for stall in (0, 1):
        ws = aw.awsrc_attention_workspace(cache, 6)
        aw.awsrc_set_wait_test(100_000_000, stall)
        try:
            aw.awsrc_paged_attention(cache, step_batch(aw, [new], [70000], table), q.cuda(), ws)
            assert aw.awsrc_workspace_status(ws) == 4
        finally:
            aw.awsrc_set_wait_test()
    check_attention(aw, cache, q, [new], [70000], table, True)


def test_graphs_with_copies_and_fills_between_the_calls(aw):
    """A captured step whose inputs are copied and outputs cleared right before each call: the calls' launches, which are
    set up early behind another kernel, wait for such nodes too. The replays give what the calls gave one by one."""
    gen = torch.Generator().manual_seed(14)
    new, kv = [1, 3, 0, 1], [700, 90, 5, 64]
    _, table, pages = make_batch(aw, gen, new, kv, 16)
    batch = step_batch(aw, new, kv, table)
    caches = [random_cache(aw, torch.Generator().manual_seed(15), pages, 2, 128, 16) for _ in range(2)]
    ws = [aw.awsrc_attention_workspace(c, 4) for c in caches]
    n = sum(new)
    src = [torch.randn(n, h, 128, generator=gen).to(BF16).cuda() for h in (4, 2, 2)]
    cos, sin = (t.cuda() for t in tables(800, 64, gen))
    q, k, v = (torch.empty_like(t) for t in src)
    out, lse = torch.empty_like(q), torch.empty(n, 4, device="cuda")

    def step(i):
        for a, b in zip((q, k, v), src):
            a.copy_(b)
        aw.awsrc_kv_append(caches[i], batch, q, k, v, cos, sin, ws[i], q_out=q)
        out.zero_()
        lse.zero_()
        aw.awsrc_paged_attention(caches[i], batch, q, ws[i], out=out, lse=lse)

    step(0)
    want = [t.clone() for t in (q, out, lse)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(1)
    for _ in range(3):
        for t in (q, k, v, out, lse):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q, out, lse), want))
    assert aw.awsrc_workspace_status(ws[1]) == 0
