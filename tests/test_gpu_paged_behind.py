"""Rows behind the last sequence of a step (n_tok above q_start[n_seq], as awsrc_kv_plan
leaves it when not all sequences find room): no call reads, writes or reports them."""
import pytest
import torch

import paged_ref as ref
from test_gpu_paged import assert_cache_equal, aw, make_batch, random_cache, tables  # noqa: F401

pytestmark = pytest.mark.gpu

I32 = torch.int32


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rotary", [0, 20, 64])
@pytest.mark.parametrize("new,behind", [([3, 4], 1), ([3, 0, 4, 0], 9), ([0, 0], 5), ([], 6), ([1] * 40, 3), ([5, 300], 70), ([1, 2600], 200)])
def test_rows_behind_the_last_sequence_are_left_alone(aw, dtype, rotary, new, behind):  # noqa: F811
    gen = torch.Generator().manual_seed(len(new) + behind)
    n, rows, page, dim = len(new), sum(new) + behind, 16, 64
    kv = [m + int(torch.randint(40, (1,), generator=gen)) for m in new]
    _, table, pages = make_batch(aw, gen, new or [1], kv or [1], page)
    base = random_cache(aw, gen, pages, 2, dim, page)
    q, k, v = (torch.randn(rows, h, dim, generator=gen).to(dtype).cuda() for h in (4, 2, 2))
    cos, sin = (t.cuda() for t in tables(max(kv + [1]), rotary // 2, gen)) if rotary else (None, None)
    start = torch.tensor([sum(new[:b]) for b in range(n + 1)], dtype=I32).cuda()
    lengths, table = torch.tensor(kv, dtype=I32).cuda(), table[:n].contiguous()

    def run(total):
        c = aw.awsrc_kv_cache(*(b.clone() for b in (base.k, base.v, base.k_exp, base.v_exp)))
        ws = aw.awsrc_attention_workspace(c, 4)
        batch = aw.awsrc_kv_batch(start, lengths, table.cuda(), total, max(new + [1]), max(kv + [1]))
        qo, out = (torch.full((total, 4, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2))
        lse = torch.full((total, 4), 7.0, device="cuda")
        aw.awsrc_kv_append(c, batch, q[:total], k[:total], v[:total], cos, sin, ws, q_out=qo)
        aw.awsrc_paged_attention(c, batch, qo, ws, out=out, lse=lse)
        assert aw.awsrc_workspace_status(ws) == 0
        return ref.Cache.of(c), qo.cpu(), out.cpu(), lse.cpu()

    live = sum(new)
    (c1, q1, o1, l1), (c0, q0, _, _) = run(rows), run(live)
    assert_cache_equal(c1, c0)
    assert torch.equal(q1[:live], q0)
    for t in (q1, o1, l1):
        assert (t[live:] == 7).all()
    # the launch's shares of the sequences may be others: against 64 bits
    eps = (2.0 ** -22, 2.0 ** -22) if dtype is torch.float32 else (0.0, 2.0 ** -9)
    want, wl, ob, lb = ref.attention(c1, q1[:live], new, kv, table, dim ** -0.5, True, *eps)
    if dtype is torch.bfloat16:
        ob = ob + (want.abs() + ob) * 2.0 ** -9  # out is rounded once
    assert ((o1[:live].double() - want).abs() <= ob + 1e-30).all() and ((l1[:live].double() - wl).abs() <= lb).all()
