"""Calls of the serving steps that are allowed and unusual: the first call of a process
inside a capture, graphs that share a workspace, maps off their vector boundaries, rows
that are one row, results of another type, plans on two streams, the most columns."""
import os
import random
import subprocess
import sys

import pytest
import torch

import step_ref as ref
from test_gpu_step_more import BF16, F32, I32, aw, cuda_ints  # noqa: F401

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST = r"""
import torch, paper_2608_23144_gb300 as aw
I32 = torch.int32
torch.manual_seed(1)
def ints(*v): return torch.tensor(v, dtype=I32).cuda()
pool = aw.awsrc_kv_pool(torch.full((2, 4), -1, dtype=I32).cuda(), ints(0, 0), torch.arange(8, dtype=I32).cuda(), ints(8), 16)
ws, add = aw.awsrc_step_workspace(), ints(20, 3)
q_start, slot = torch.zeros(3, dtype=I32, device="cuda"), torch.zeros(24, dtype=torch.int64, device="cuda")
p = torch.softmax(torch.randn(5, 200, device="cuda"), -1)
starts, ids, u, r = ints(0, 3, 5), ints(1, 2, 3, 4, 5), torch.rand(5, device="cuda"), torch.rand(2, device="cuda")
acc, tok = torch.empty(2, dtype=I32, device="cuda"), torch.empty(2, 3, dtype=I32, device="cuda")
w, xs = torch.randn(3000, 900, device="cuda"), [torch.randn(m, 900, device="cuda") for m in (1, 16, 40, 200)]
w8, x8 = aw.awsrc_fp8_matrix(3000, 900), [aw.awsrc_fp8_matrix(x.shape[0], 900) for x in xs]
ys = [torch.empty(x.shape[0], 3000, device="cuda") for x in xs]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):  # nothing of the library has run but the workspace's fill
    aw.awsrc_kv_plan(pool, None, add, ws, q_start=q_start, tok_slot=slot)
    aw.awsrc_verify_drafts(starts, ids, p, None, u, r, ws, accepted=acc, tokens=tok)
    aw.awsrc_fp8_quantize(w, out=w8)
    for x, m, y in zip(xs, x8, ys):
        aw.awsrc_fp8_linear(x, w8, m, ws, out=y)
graph.replay()
torch.cuda.synchronize()
assert q_start.tolist() == [0, 20, 23] and pool.free_count.item() == 5 and slot[:17].tolist() == [*range(112, 128), 96]
want = aw.awsrc_verify_drafts(starts, ids, p, None, u, r, ws, max_draft=2)
assert torch.equal(acc, want[0]) and torch.equal(tok, want[1])
for x, y in zip(xs, ys):
    assert torch.equal(y, aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), aw.awsrc_fp8_quantize(w), ws))
assert aw.awsrc_workspace_status(ws) == 0
print("right")
"""


def test_first_calls_of_a_process_inside_a_capture():
    r = subprocess.run([sys.executable, "-c", FIRST], cwd=ROOT,
                       env=dict(os.environ, PYTHONPATH=ROOT), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "right", (r.stdout, r.stderr[-2000:])


def test_graphs_that_share_a_workspace(aw):  # noqa: F811
    """A plan and a product captured into two graphs with one workspace, replayed in turn on one stream."""
    gen = torch.Generator().manual_seed(2)
    ws, side = aw.awsrc_step_workspace(), torch.cuda.Stream()
    pool = aw.awsrc_kv_pool(torch.full((5, 9), -1, dtype=I32).cuda(), cuda_ints([0] * 5), torch.arange(45, dtype=I32).cuda(),
                            cuda_ints([45]), 16)
    add, slot = cuda_ints([3, 1, 4, 1, 5]), torch.zeros(14, dtype=torch.int64, device="cuda")
    q_start = torch.zeros(6, dtype=I32, device="cuda")
    w = aw.awsrc_fp8_quantize(torch.randn(2000, 640, generator=gen).cuda())
    sets = [(torch.randn(m, 640, generator=gen).cuda(), aw.awsrc_fp8_matrix(m, 640), torch.empty(m, 2000, device="cuda")) for m in (5, 90)]
    want = [aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), w, ws) for x, _, _ in sets]
    graphs = []
    torch.cuda.synchronize()
    for x, x8, y in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            aw.awsrc_kv_plan(pool, None, add, ws, q_start=q_start, tok_slot=slot)
            aw.awsrc_fp8_linear(x, w, x8, ws, out=y)
    length = [0] * 5
    for i in range(8):
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        length = [k + a for k, a in zip(length, add.tolist())]
        assert pool.kv_len.tolist() == length and torch.equal(sets[i % 2][2], want[i % 2])
    assert slot.min() >= 0 and slot.unique().numel() == 14 and aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("which", [(0, 1, 2), (0,), (1,), (2,), (0, 2), (1, 2)])
@pytest.mark.parametrize("off", [0, 1, 2, 3])
def test_plan_maps_off_their_boundaries(aw, which, off):  # noqa: F811
    """Some of the maps, starting anywhere in wider tensors; the elements around them stay."""
    rng = random.Random(off)
    lengths, add, n_tok, page = [5, 0, 33, 16], [3, 17, 1, 0], 27, 16
    table = [[-1] * 6 for _ in range(4)]
    pages, at = list(range(20)), 0
    rng.shuffle(pages)
    for b, k in enumerate(lengths):
        for j in range(-(-k // page)):
            table[b][j] = pages[at]
            at += 1
    free = pages[at:] + [-1] * at
    want = ref.plan(page, table, lengths, free, 20 - at, None, add, n_tok)
    pool = aw.awsrc_kv_pool(cuda_ints(table), cuda_ints(lengths), cuda_ints(free), cuda_ints([20 - at]), page)
    wide = [torch.full((n_tok + 8,), 77, dtype=t, device="cuda") for t in (I32, I32, torch.int64)]
    maps = [wide[i][off:off + n_tok] if i in which else None for i in range(3)]
    q = aw.awsrc_kv_plan(pool, None, cuda_ints(add), aw.awsrc_step_workspace(), n_tok=n_tok, tok_seq=maps[0], tok_pos=maps[1],
                         tok_slot=maps[2])
    assert q.tolist() == want[4]
    for i, (m, full) in enumerate(zip(maps, wide)):
        if m is not None:
            assert m.tolist() == want[5 + i]
        assert (full[:off] == 77).all() and (full[off + (n_tok if m is not None else 0):] == 77).all()


def test_rows_that_are_one_row(aw):  # noqa: F811
    """Expanded tensors (row stride 0) of probabilities and of activations, one column, a single row of any stride."""
    gen = torch.Generator().manual_seed(6)
    p = torch.softmax(torch.randn(1, 300, generator=gen), -1)
    ws, n = aw.awsrc_step_workspace(), 7
    u, r, ids = torch.rand(n, generator=gen).cuda(), torch.rand(n, generator=gen).cuda(), cuda_ints([3] * n)
    starts = torch.arange(n + 1, dtype=I32).cuda()
    for q in (None, p.flip(1)):
        a = aw.awsrc_verify_drafts(starts, ids, p.cuda().expand(n, 300), None if q is None else q.cuda().expand(n, 300), u, r, ws, max_draft=0)
        b = aw.awsrc_verify_drafts(starts, ids, p.repeat(n, 1).cuda(), None if q is None else q.repeat(n, 1).cuda(), u, r, ws, max_draft=0)
        assert torch.equal(a[1], b[1]) and (a[1] >= 0).all()
    for m, k in ((1, 700), (5, 700), (90, 700), (1, 1), (30, 1)):
        x = torch.randn(1, k, generator=gen).cuda()
        w = aw.awsrc_fp8_quantize(torch.randn(333, k, generator=gen).cuda())
        y = aw.awsrc_fp8_linear(x.expand(m, k), w, aw.awsrc_fp8_matrix(m, k), ws)
        assert torch.equal(y, aw.awsrc_fp8_linear(x.repeat(m, 1), w, aw.awsrc_fp8_matrix(m, k), ws)) and torch.equal(y[:1].expand(m, 333), y)
    assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("m", [1, 2, 16, 40, 100])
@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, BF16), (BF16, F32)])
def test_results_of_another_type_than_x(aw, m, x_dtype, y_dtype):  # noqa: F811
    gen = torch.Generator().manual_seed(m)
    x, w = torch.randn(m, 1000, generator=gen).to(x_dtype).cuda(), aw.awsrc_fp8_quantize(torch.randn(700, 1000, generator=gen).cuda())
    ws, x8 = aw.awsrc_step_workspace(), aw.awsrc_fp8_matrix(m, 1000)
    y = aw.awsrc_fp8_linear(x, w, x8, ws, out=torch.empty(m, 700, dtype=y_dtype, device="cuda"))
    assert torch.equal(y, aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), w, ws, out_dtype=y_dtype))


def test_plans_and_verifications_on_two_streams(aw):  # noqa: F811
    """Each with its own pool and workspace, 60 times over."""
    gen = torch.Generator().manual_seed(9)
    sets = []
    for n in (9, 700):
        pool = aw.awsrc_kv_pool(torch.full((n, 20), -1, dtype=I32).cuda(), cuda_ints([0] * n), torch.arange(20 * n, dtype=I32).cuda(),
                                cuda_ints([20 * n]), 16)
        p = torch.softmax(torch.randn(2 * n, 900, generator=gen), -1).cuda()
        sets.append((n, pool, aw.awsrc_step_workspace(), torch.full((n,), 4, dtype=I32, device="cuda"), torch.zeros(n + 1, dtype=I32, device="cuda"),
                     torch.zeros(4 * n, dtype=torch.int64, device="cuda"), p, torch.arange(0, 2 * n + 1, 2, dtype=I32).cuda(),
                     torch.randint(900, (2 * n,), generator=gen).to(I32).cuda(), torch.rand(2 * n, generator=gen).cuda(),
                     torch.rand(n, generator=gen).cuda(), torch.empty(n, dtype=I32, device="cuda"), torch.empty(n, 2, dtype=I32, device="cuda")))
    want = [aw.awsrc_verify_drafts(s[7], s[8], s[6], None, s[9], s[10], s[2], max_draft=1) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(60):
        for (n, pool, ws, add, q, slot, p, st, ids, u, r, acc, tok), s in zip(sets, streams):
            aw.awsrc_kv_plan(pool, None, add, ws, q_start=q, tok_slot=slot, stream=s)
            aw.awsrc_verify_drafts(st, ids, p, None, u, r, ws, accepted=acc, tokens=tok, stream=s)
    torch.cuda.synchronize()
    for (n, pool, ws, *_, acc, tok), w in zip(sets, want):
        assert pool.kv_len.tolist() == [240] * n and pool.free_count.item() == 5 * n
        held = pool.page_table[:, :15].flatten().tolist() + pool.free_pages[:5 * n].tolist()
        assert sorted(held) == list(range(20 * n)) and torch.equal(acc, w[0]) and torch.equal(tok, w[1])
        assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("m", [1, 20, 70])
def test_the_most_columns(aw, m):  # noqa: F811
    """2^24 columns, ones here and there in the first, the middle and the last blocks."""
    k, n = 1 << 24, 9
    at = torch.tensor([0, 127, 128, 511, 512, 32767, 32768, k // 2 - 1, k // 2, k // 3, k - 129, k - 128, k - 1], device="cuda")
    x, w = (torch.zeros(r, k, dtype=BF16, device="cuda") for r in (m, n))
    x[:, at] = (torch.arange(m * 13, device="cuda").view(m, 13) % 7 - 3).to(BF16)
    w[:, at] = (torch.arange(n * 13, device="cuda").view(n, 13) % 5 - 2).to(BF16)
    want = x[:, at].float() @ w[:, at].float().T
    ws = aw.awsrc_step_workspace()
    y = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), aw.awsrc_fp8_quantize(w), ws)
    assert torch.equal(y, want) and aw.awsrc_workspace_status(ws) == 0
    torch.cuda.empty_cache()


def test_verify_the_most_sequences(aw):  # noqa: F811
    """65535 sequences of one row each: the token is the first whose running sum of units is above r of them all."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    n, vocab = 65535, 37
    p = torch.rand(n, vocab, generator=gen, device="cuda") / 64
    k = torch.randint(256, (n,), generator=gen, device="cuda")  # r = k / 256
    sums = torch.round(p.double() * 2.0 ** 45).long().cumsum(1)  # float32 below 2^-6 in units of 2^-45: exact but for their last bits
    want = (sums * 256 <= k[:, None] * sums[:, -1:]).sum(1)
    ws = aw.awsrc_step_workspace()
    starts, ids = torch.arange(n + 1, dtype=I32, device="cuda"), torch.zeros(n, dtype=I32, device="cuda")
    acc, tok = aw.awsrc_verify_drafts(starts, ids, p, None, torch.zeros(n, device="cuda"), k.float() / 256, ws, max_draft=0)
    assert torch.equal(tok[:, 0].long(), want) and not acc.any() and aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("stop", [0, 1, 31, 1024, 2999, 3000])
def test_verify_thousands_of_drafts(aw, stop):  # noqa: F811
    """3000 drafts of one sequence beside one of none: accepted up to the first whose random number refuses it."""
    gen = torch.Generator().manual_seed(stop)
    drafts, vocab = 3000, 20
    p = torch.softmax(torch.randn(drafts + 2, vocab, generator=gen) * 2, -1)
    ids = torch.randint(vocab, (drafts + 2,), generator=gen)
    u = torch.zeros(drafts + 2)
    u[stop:] = 1.0
    ws = aw.awsrc_step_workspace()
    acc, tok = aw.awsrc_verify_drafts(cuda_ints([0, drafts + 1, drafts + 2]), ids.to(I32).cuda(), p.cuda(), None, u.cuda(),
                                      torch.tensor([0.4, 0.6]).cuda(), ws, max_draft=drafts + 5)
    assert acc.tolist() == [stop, 0] and tok.shape == (2, drafts + 6)
    assert tok[0, :stop].tolist() == ids[1:stop + 1].tolist() and (tok[0, stop + 1:] == -1).all() and (tok[1, 1:] == -1).all()
    rows = ref.verify([0, 1], [0], p[stop:stop + 1].double().tolist(), None, [0.0], [0.4], 0, [9])[1][0][0] if stop == drafts else None
    assert 0 <= tok[0, stop] < vocab and (tok[0, stop] == rows if rows is not None else tok[0, stop] != ids[stop + 1])
    assert aw.awsrc_workspace_status(ws) == 0
