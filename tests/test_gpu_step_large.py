"""Serving-step calls whose offsets pass 32 bits: matrices of more than 2^31 bytes of
codes, results and rows of probabilities of more than 2^31 elements, slots of pages
whose numbers times their size pass 2^31."""
import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def aw():
    import paper_2608_23144_gb300 as aw
    assert torch.cuda.is_available()
    yield aw
    torch.cuda.empty_cache()


def test_matrices_of_more_than_2_31_codes(aw):
    rows, k, last = 1_100_000, 2048, 300
    gen = torch.Generator(device="cuda").manual_seed(1)
    big = torch.randn(rows, k, generator=gen, device="cuda", dtype=BF16)
    m = aw.awsrc_fp8_quantize(big)
    end = aw.awsrc_fp8_quantize(big[rows - last:])
    assert m.codes.numel() > 2 ** 31
    small = aw.awsrc_fp8_quantize(torch.randn(3, k, generator=gen, device="cuda"))
    ws = aw.awsrc_step_workspace()
    del big
    want = small.values().double() @ end.values().double().T
    y = aw.awsrc_fp8_gemm(small, m, ws)[:, rows - last:].double()  # the weights' rows
    assert (y - want).norm() <= 1e-5 * want.norm()
    other = aw.awsrc_fp8_quantize(torch.randn(40, k, generator=gen, device="cuda"))
    y = aw.awsrc_fp8_gemm(m, other, ws)[rows - last:].double()  # the activations' rows
    want = end.values().double() @ other.values().double().T
    assert (y - want).norm() <= 1e-5 * want.norm()
    assert aw.awsrc_workspace_status(ws) == 0


def test_results_of_more_than_2_31_elements(aw):
    rows, cols = 70_001, 31_000
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = aw.awsrc_fp8_quantize(torch.randn(rows, 128, generator=gen, device="cuda"))
    w = aw.awsrc_fp8_quantize(torch.randn(cols, 128, generator=gen, device="cuda"))
    y = aw.awsrc_fp8_gemm(x, w, aw.awsrc_step_workspace(), out_dtype=BF16)
    assert y.numel() > 2 ** 31
    for a in (0, rows - 130):
        want = x.values()[a:a + 130].double() @ w.values().double().T
        assert (y[a:a + 130].double() - want).norm() <= 2.0 ** -8 * want.norm()


def test_a_row_stride_that_passes_32_bits(aw):
    gen = torch.Generator(device="cuda").manual_seed(3)
    wide = torch.empty(3, 1_500_000_000, dtype=BF16, device="cuda")
    x = wide[:, 5:645]
    x.copy_(torch.randn(3, 640, generator=gen, device="cuda"))
    w = aw.awsrc_fp8_quantize(torch.randn(200, 640, generator=gen, device="cuda"))
    ws, x8 = aw.awsrc_step_workspace(), aw.awsrc_fp8_matrix(3, 640)
    out = wide[:, 1_400_000_000:1_400_000_200]
    aw.awsrc_fp8_linear(x, w, x8, ws, out=out)
    want = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x.contiguous()), w, ws, out_dtype=BF16)
    assert torch.equal(out, want)


def test_rows_of_probabilities_past_2_31(aw):
    rows, vocab = 17_000, 130_000
    gen = torch.Generator(device="cuda").manual_seed(4)
    p = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    assert p.numel() > 2 ** 31
    at = rows - 4
    p[at:] = torch.softmax(torch.randn(4, vocab, generator=gen, device="cuda") * 3, -1).to(BF16)
    ids = torch.zeros(rows, dtype=I32, device="cuda")
    ids[at + 1:] = p[at:rows - 1].argmax(-1)
    u, r = torch.full((rows,), 0.01, device="cuda"), torch.tensor([0.3, 0.9], device="cuda")
    acc, tok = aw.awsrc_verify_drafts(torch.tensor([at, at + 2, rows], dtype=I32, device="cuda"), ids, p, None, u, r,
                                      aw.awsrc_step_workspace(), max_draft=1)
    want = ref.verify([0, 2, 4], ids[at:].tolist(), p[at:].double().tolist(), None, u[at:].tolist(), r.tolist(), 1, [9, 9])
    assert acc.tolist() == want[0] and tok.tolist() == want[1]


def test_slots_past_2_31(aw):
    pages = 1 << 26  # of 128 tokens: slots up to 2^33
    free = torch.full((pages,), -1, dtype=I32, device="cuda")
    free[:3] = torch.tensor([pages - 1, pages - 2, pages - 3])
    table = torch.tensor([[pages - 4, -1, -1], [pages - 5, -1, -1]], dtype=I32, device="cuda")
    pool = aw.awsrc_kv_pool(table, torch.tensor([127, 5], dtype=I32, device="cuda"), free,
                            torch.tensor([3], dtype=I32, device="cuda"), 128)
    slot = torch.empty(4, dtype=torch.int64, device="cuda")
    aw.awsrc_kv_plan(pool, None, torch.tensor([3, 1], dtype=I32, device="cuda"), aw.awsrc_step_workspace(), tok_slot=slot)
    assert slot.tolist() == [(pages - 4) * 128 + 127, (pages - 3) * 128, (pages - 3) * 128 + 1, (pages - 5) * 128 + 5]
    assert pool.free_count.item() == 2
