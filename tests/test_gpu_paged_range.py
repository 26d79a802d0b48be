"""The paged cache over the ranges of its inputs: what queries, marks, scales and
batches may hold, beside the sizes of test_gpu_paged.py. The references and the
derived bounds are those of paged_ref.py."""
import pytest
import torch

import paged_ref as ref
from test_gpu_paged import BF16, F32, aw, check_attention, make_batch, random_cache, step_batch, tables  # noqa: F401

pytestmark = pytest.mark.gpu

BF16_EPS = (0.0, 2.0 ** -11)  # q exact, weights in one binary16
BF16_ROUND = 2.0 ** -8  # out, once, to 8 significant bits: half a unit of the last, 2^-8 of a power of two


# ------------------------------------------------------------------ queries

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(6, 2, 128), (3, 3, 64)])
@pytest.mark.parametrize("new", [1, 40, 300])
@pytest.mark.parametrize("ratio", [2.0 ** 8, 2.0 ** 11, 2.0 ** 14])
def test_a_query_channel_far_above_the_others(aw, dtype, heads, kv_heads, dim, new, ratio):  # noqa: F811
    """One dim of every query is `ratio` times the others and meets keys of zero there, so that the scores come from the
    small dims alone. The bounds of paged_ref.py take q as exact (BF16) or to 2^-22 of each element (float32). BF16 with
    more than 16 rows per kv head adds an error of 2^-21 of a row's largest element for elements below 2^-13 of it: dx
    in a score, so dx (relative) in the softmax sum and 2 dx sum_j p_j |v_j| in out."""
    gen = torch.Generator().manual_seed(20)
    kv = [max(new, 333)]
    _, table, pages = make_batch(aw, gen, [new], kv, 32)
    cache = random_cache(aw, gen, pages, kv_heads, dim, 32)
    cache.k.view(torch.uint8)[:, :, 2, :, 5] = 0  # dim 37
    q = torch.randn(new, heads, dim, generator=gen)
    q[..., 37] = torch.where(q[..., 37] < 0, -ratio, ratio)
    q = q.to(dtype)
    if dtype == F32 or new * heads // kv_heads <= 16:
        check_attention(aw, cache, q, [new], kv, table, True)
        return
    c = ref.Cache.of(cache)
    want, wl, ob, lb = ref.attention(c, q, [new], kv, table, dim ** -0.5, True, *BF16_EPS)
    x = q.double().abs()
    top = x.amax(-1, keepdim=True)
    small = torch.where(x < top * 2.0 ** -13, top * 2.0 ** -21, 0.0)
    used = [int(p) for p in table[0][:-(-kv[0] // 32)]]
    for h in range(heads):
        k, v = (c.values(w, used, h // (heads // kv_heads), kv[0]) for w in "kv")
        hide = torch.arange(kv[0])[None] > (kv[0] - new + torch.arange(new))[:, None]
        dx = (small[:, h] @ k.abs().T * dim ** -0.5).masked_fill(hide, 0.0).amax(1)
        p = torch.softmax((q[:, h].double() @ k.T * dim ** -0.5).masked_fill(hide, -torch.inf), 1)
        ob[:, h] += 2 * dx[:, None] * (p @ v.abs())
        lb[:, h] += dx
    lse = torch.empty(new, heads, device="cuda")
    out = aw.awsrc_paged_attention(cache, step_batch(aw, [new], kv, table), q.cuda(),
                                   aw.awsrc_attention_workspace(cache, heads), lse=lse).cpu().double()
    assert ((out - want).abs() <= ob + (want.abs() + ob) * BF16_ROUND).all()  # out is rounded once
    assert ((lse.cpu().double() - wl).abs() <= lb).all()


# -------------------------------------------------------------------- marks

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,kv,page", [(1, 300, 16), (40, 300, 16), (40, 300, 64), (1, 9000, 32), (40, 9000, 128)])
def test_marked_blocks(aw, dtype, which, dim, new, kv, page):  # noqa: F811
    """A block marked as not finite reaches the queries and heads that see it, and no others. Marked keys: scores, so out
    and lse, are NaN. Marked values: out is NaN, but the scores and lse are what they were."""
    gen = torch.Generator().manual_seed(21)
    _, table, pages = make_batch(aw, gen, [new], [kv], page)
    cache = random_cache(aw, gen, pages, 2, dim, page)
    slot = (kv - 20) // page  # some of 40 queries end before it (pages of 16), some do not
    pg = int(table[0, slot])
    q = torch.randn(new, 6, dim, generator=gen).to(dtype)
    ws = aw.awsrc_attention_workspace(cache, 6)
    batch = step_batch(aw, [new], [kv], table)
    eps = (2.0 ** -22, 2.0 ** -22) if dtype == F32 else BF16_EPS
    want, wl, ob, lb = ref.attention(ref.Cache.of(cache), q, [new], [kv], table, dim ** -0.5, True, *eps)
    if dtype == BF16:
        ob = ob + (want.abs() + ob) * BF16_ROUND
    (cache.k_exp if which == "k" else cache.v_exp)[pg, 1] = -128
    lse = torch.empty(new, 6, device="cuda")
    out = aw.awsrc_paged_attention(cache, batch, q.cuda(), ws, lse=lse).cpu().double()
    lse = lse.cpu().double()
    assert aw.awsrc_workspace_status(ws) == 0
    hit = (torch.arange(kv - new, kv) >= slot * page)[:, None] & (torch.arange(6) >= 3)[None]
    assert torch.equal(torch.isnan(out).all(-1), hit) and torch.equal(torch.isnan(out).any(-1), hit)
    assert ((out - want).abs() <= ob + 1e-30)[~hit].all()
    if which == "k":
        assert torch.equal(torch.isnan(lse), hit)
    ok = ~hit if which == "k" else torch.ones_like(hit)
    assert ((lse - wl).abs() <= lb)[ok].all()


# ------------------------------------------------------------------ batches

@pytest.mark.parametrize("n_seq,at", [(20, 17), (130, 128), (300, 290)])
@pytest.mark.parametrize("kind", ["negative length", "length beyond the table", "falling start"])
def test_append_reports_every_entry_that_cannot_be_right(aw, n_seq, at, kind):  # noqa: F811
    """Bad entries without rows of their own, in any place of the batch; the sequences that overlap no bad entry's rows
    get what they get without it."""
    gen = torch.Generator().manual_seed(22)
    page, heads, dim = 16, 2, 64
    new, kv = [2] * n_seq, [37] * n_seq
    new[at] = 0
    _, table, pages = make_batch(aw, gen, new, kv, page)
    base = random_cache(aw, gen, pages, heads, dim, page)
    n = sum(new)
    x = torch.randn(3, n, heads, dim, generator=gen).cuda()
    start = [sum(new[:b]) for b in range(n_seq + 1)]

    def run(start, kv):
        c = aw.awsrc_kv_cache(*(b.clone() for b in (base.k, base.v, base.k_exp, base.v_exp)))
        ws = aw.awsrc_attention_workspace(c, heads)
        batch = aw.awsrc_kv_batch(torch.tensor(start, dtype=torch.int32).cuda(), torch.tensor(kv, dtype=torch.int32).cuda(),
                                  table.cuda(), n, 4, 48)
        aw.awsrc_kv_append(c, batch, *x, None, None, ws)
        return c, aw.awsrc_workspace_status(ws)

    good, flags = run(start, kv)
    assert flags == 0
    start, kv = list(start), list(kv)
    if kind == "negative length":
        kv[at] = -1
    elif kind == "length beyond the table":
        kv[at] = page * table.shape[1] + 1
    else:  # entry `at` ends before it starts, so that the one behind it takes two rows of the one before it
        start[at + 1] -= 2
    got, flags = run(start, kv)
    assert flags == 8
    same = [b for b in range(n_seq) if b not in (at, at + 1)]
    pg = table[same].long().cuda().flatten()
    for a, b in ((got.k, good.k), (got.v, good.v)):
        assert torch.equal(a.view(torch.uint8)[pg], b.view(torch.uint8)[pg])
    assert torch.equal(got.k_exp[pg], good.k_exp[pg]) and torch.equal(got.v_exp[pg], good.v_exp[pg])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seq", [33, 129, 300])
@pytest.mark.parametrize("most", [1, 9])
def test_batches_of_many_sequences(aw, dtype, n_seq, most):  # noqa: F811
    """More sequences than a warp, a thread block and two of them look at together, some without new tokens and some
    empty: appended bit for bit, then read by the kernel of few rows (one token each) and by that of many."""
    gen = torch.Generator().manual_seed(n_seq)
    heads, kv_heads, dim, page = 6, 2, 64, 16
    new = torch.randint(0, most + 1, (n_seq,), generator=gen)
    ctx = torch.randint(0, 60, (n_seq,), generator=gen) * (torch.rand(n_seq, generator=gen) < 0.8)
    kv = (new + ctx).tolist()
    new = new.tolist()
    batch, table, pages = make_batch(aw, gen, new, kv, page)
    cache = random_cache(aw, gen, pages, kv_heads, dim, page)
    want = ref.Cache.of(cache)
    ws = aw.awsrc_attention_workspace(cache, heads)
    x = torch.randn(sum(new), heads + 2 * kv_heads, dim, generator=gen).to(dtype)
    cos, sin = tables(max(kv), dim // 2, gen)
    cut = (slice(0, heads), slice(heads, heads + kv_heads), slice(heads + kv_heads, None))
    q = aw.awsrc_kv_append(cache, batch, *(x.cuda()[:, c] for c in cut), cos.cuda(), sin.cuda(), ws)
    assert aw.awsrc_workspace_status(ws) == 0
    want_q = ref.append(want, *(x[:, c] for c in cut), new, kv, table, cos, sin, False)
    assert torch.equal(q.cpu(), want_q.to(dtype))
    got = ref.Cache.of(cache)
    for w in "kv":
        assert torch.equal(got.exp[w], want.exp[w]) and torch.equal(got.code[w], want.code[w])
    check_attention(aw, cache, q.cpu(), new, kv, table, True, batch=batch, ws=ws)


# ------------------------------------------------------------------- scales

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("scale", [0.0, -0.11, 1e-30])
def test_score_scales_of_either_sign_and_zero(aw, dtype, new, scale):  # noqa: F811
    """sm_scale q and |sm_scale| (-q) are the same scores, and the bounds are those of the second."""
    gen = torch.Generator().manual_seed(23)
    kv = [new + 211]
    _, table, pages = make_batch(aw, gen, [new], kv, 16)
    cache = random_cache(aw, gen, pages, 2, 128, 16)
    q = torch.randn(new, 6, 128, generator=gen).to(dtype)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty(new, 6, device="cuda")
    ws = aw.awsrc_attention_workspace(cache, 6)
    aw.awsrc_paged_attention(cache, step_batch(aw, [new], kv, table), q.cuda(), ws, sm_scale=scale, out=out, lse=lse)
    eps = (2.0 ** -22, 2.0 ** -22) if dtype == F32 else BF16_EPS
    want, wl, ob, lb = ref.attention(ref.Cache.of(cache), -q if scale < 0 else q, [new], kv, table, abs(scale), True, *eps)
    if dtype == BF16:
        ob = ob + (want.abs() + ob) * BF16_ROUND
    assert ((out.cpu().double() - want).abs() <= ob + 1e-30).all()
    assert ((lse.cpu().double() - wl).abs() <= lb).all()


# ------------------------------------------------------------------ weights

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,kv", [(1, 200), (40, 200), (40, 5000)])
@pytest.mark.parametrize("spread", [8, 16, 24])
def test_values_of_one_block_far_above_the_others(aw, dtype, new, kv, spread):  # noqa: F811
    """One block's value scale is 2^spread times the others', for the sake of one dim; its other dims are zero, so that the
    rest of the output comes from weights that count 2^-spread as much. A weight times its scale is held to 2^-22
    (float32) or 2^-11 of itself, or to W 2^-40 (tiles kernel: 2^-31), W the row's largest: sum_j |c_j| W 2^-40 more in out."""
    gen = torch.Generator().manual_seed(24)
    page, dim, heads = 16, 64, 6
    _, table, pages = make_batch(aw, gen, [new], [kv], page)
    cache = random_cache(aw, gen, pages, 1, dim, page)
    cache.k_exp.fill_(-9)
    cache.v_exp.fill_(-12)
    big = int(table[0, 5])
    cache.v_exp[big] = spread - 12
    raw = cache.v.view(torch.uint8)
    raw[big, :, :, :7] = 0
    raw[big, :, :, 8:] = 0  # dim 7 alone
    q = torch.randn(new, heads, dim, generator=gen).to(dtype)
    c = ref.Cache.of(cache)
    tiles = dtype == BF16 and new * heads > 16
    eps = (2.0 ** -22, 2.0 ** -22) if dtype == F32 else BF16_EPS
    want, wl, ob, lb = ref.attention(c, q, [new], [kv], table, dim ** -0.5, True, *eps)
    used = [int(p) for p in table[0][:-(-kv // page)]]
    k, v = (c.values(w, used, 0, kv) for w in "kv")
    scale = torch.exp2(c.exp["v"][used, 0].double()).repeat_interleave(page)[:kv]
    hide = torch.arange(kv)[None] > (kv - new + torch.arange(new))[:, None]
    for h in range(heads):
        p = torch.softmax((q[:, h].double() @ k.T * dim ** -0.5).masked_fill(hide, -torch.inf), 1)
        codes = (v / scale[:, None]).abs()
        ob[:, h] += 2.0 ** (-31 if tiles else -40) * (p * scale).amax(1, keepdim=True) * ((~hide).double() @ codes)
    if dtype == BF16:
        ob = ob + (want.abs() + ob) * BF16_ROUND
    lse = torch.empty(new, heads, device="cuda")
    out = aw.awsrc_paged_attention(cache, step_batch(aw, [new], [kv], table), q.cuda(),
                                   aw.awsrc_attention_workspace(cache, heads), lse=lse).cpu().double()
    assert ((out - want).abs() <= ob).all()
    assert ((lse.cpu().double() - wl).abs() <= lb).all()
