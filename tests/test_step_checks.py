"""What the serving-step calls refuse before any launch, at the C boundary (status
codes) and in the Python binding (exceptions). No GPU: pointers are made-up numbers,
tensors live on the CPU, and every call must stop at a check."""
import ctypes as ct

import pytest
import torch

import paper_2608_23144_gb300 as aw
from paper_2608_23144_gb300 import _step

OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 6  # awsrc_status

P = 1 << 20  # an aligned address that nothing reads


def pool(**over):
    c = dict(n_pages=8, page=64, n_seq=2, table_stride=4, page_table=P, kv_len=P, free_pages=P, free_count=P)
    c.update(over)
    return _step._Pool(**c)


def plan(p=None, keep=P, add=P, n_tok=0, q_start=P, seq=None, pos=None, slot=None, ws=P, ws_bytes=1 << 30):
    return aw.lib.awsrc_kv_plan(ct.byref(p or pool()), keep, add, n_tok, q_start, seq, pos, slot, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(p=pool(n_pages=0)), INVALID), (dict(p=pool(n_seq=-1)), INVALID), (dict(p=pool(table_stride=0)), INVALID),
    (dict(p=pool(page=48)), SHAPE), (dict(p=pool(page=0)), SHAPE), (dict(p=pool(n_seq=8193)), UNSUPPORTED),
    (dict(p=pool(table_stride=(1 << 24) + 1)), UNSUPPORTED), (dict(p=pool(page_table=None)), INVALID),
    (dict(p=pool(kv_len=None)), INVALID), (dict(p=pool(free_pages=P + 2)), INVALID), (dict(p=pool(free_count=None)), INVALID),
    (dict(add=None), INVALID), (dict(keep=P + 1), INVALID), (dict(n_tok=-1), INVALID), (dict(q_start=None), INVALID),
    (dict(seq=P + 2), INVALID), (dict(pos=P + 1), INVALID), (dict(slot=P + 4), INVALID), (dict(ws=None), WORKSPACE),
    (dict(ws_bytes=255), WORKSPACE), (dict(ws=P + 16), INVALID), (dict(p=pool(n_pages=(1 << 30) + 1)), UNSUPPORTED),
    (dict(n_tok=(1 << 30) + 1), UNSUPPORTED),
])
def test_plan_refuses(kw, status):
    assert plan(**kw) == status


def test_plan_refuses_the_lengths_themselves_as_keep():
    """With keep in kv_len's place nothing says what a sequence held before."""
    assert plan(p=pool(kv_len=2 * P), keep=2 * P) == INVALID


def probs(**over):
    c = dict(p=P, stride=100, dtype=0, pad_=0)
    c.update(over)
    return _step._Probs(**c)


def verify(n_seq=0, n_rows=5, vocab=100, max_draft=3, start=P, ids=P, p=None, q=None, u=P, r=P, kv=P, acc=P, tok=P, keep=P, ws=P,
           ws_bytes=1 << 30):
    return aw.lib.awsrc_verify_drafts(n_seq, n_rows, vocab, max_draft, start, ids, ct.byref(p or probs()),
                                      ct.byref(q) if q else None, u, r, kv, acc, tok, keep, ws, ws_bytes, None)


def test_verification_of_no_sequences_passes():
    assert verify() == OK and verify(q=probs(dtype=1)) == OK and verify(kv=None, keep=None) == OK


@pytest.mark.parametrize("kw,status", [
    (dict(n_seq=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(max_draft=-1), INVALID), (dict(vocab=0), SHAPE),
    (dict(n_seq=65536), UNSUPPORTED), (dict(vocab=(1 << 18) + 1), UNSUPPORTED), (dict(max_draft=(1 << 20) + 1), UNSUPPORTED),
    (dict(start=None), INVALID), (dict(ids=P + 2), INVALID), (dict(p=probs(p=None)), INVALID), (dict(p=probs(dtype=2)), INVALID),
    (dict(p=probs(p=P + 2)), INVALID), (dict(q=probs(dtype=3)), INVALID), (dict(q=probs(dtype=1, p=P + 1)), INVALID),
    (dict(u=None), INVALID), (dict(r=P + 1), INVALID), (dict(kv=None), INVALID), (dict(keep=None), INVALID),
    (dict(acc=None), INVALID), (dict(tok=P + 3), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(ws=P + 64), INVALID),
])
def test_verification_refuses(kw, status):
    assert verify(**kw) == status


def mat(**over):
    c = dict(rows=0, cols=256, codes=P, exps=P)
    c.update(over)
    return _step._Fp8(**c)


def gemm(x=None, w=None, y=P, dtype=0, stride=10, ws=P, ws_bytes=1 << 30):
    return aw.lib.awsrc_fp8_gemm(ct.byref(x or mat()), ct.byref(w or mat(rows=10, codes=2 * P, exps=2 * P)), y, dtype, stride, ws, ws_bytes, None)


def linear(x=None, w=None, y=P, dtype=0, stride=10, ws=P, ws_bytes=1 << 30, src=P, src_dtype=0):
    return aw.lib.awsrc_fp8_linear(src, src_dtype, 256, ct.byref(x or mat()),
                                   ct.byref(w or mat(rows=10, codes=2 * P, exps=2 * P)), y, dtype, stride, ws, ws_bytes, None)


def quantize(src=P, dtype=0, stride=256, out=None):
    return aw.lib.awsrc_fp8_quantize(src, dtype, stride, ct.byref(out or mat()), None)


def test_products_without_rows_pass():
    assert gemm() == OK and linear() == OK and quantize() == OK
    assert gemm(x=mat(rows=4), w=mat()) == OK


@pytest.mark.parametrize("call", [gemm, linear])
@pytest.mark.parametrize("kw,status", [
    (dict(x=mat(rows=-1)), INVALID), (dict(x=mat(cols=0)), SHAPE), (dict(w=mat(rows=(1 << 30) + 1)), UNSUPPORTED),
    (dict(w=mat(cols=(1 << 24) + 1)), UNSUPPORTED), (dict(x=mat(codes=None)), INVALID), (dict(w=mat(exps=None)), INVALID),
    (dict(x=mat(codes=P + 64)), INVALID), (dict(w=mat(exps=P + 8)), INVALID), (dict(w=mat(cols=128)), SHAPE),
    (dict(y=None), INVALID), (dict(y=P + 2), INVALID), (dict(dtype=2), INVALID), (dict(ws=None), WORKSPACE),
    (dict(ws_bytes=255), WORKSPACE), (dict(ws=P + 128), INVALID),
    (dict(x=mat(rows=1 << 30), w=mat(rows=1 << 30), stride=1 << 30), UNSUPPORTED),
    (dict(x=mat(rows=2), stride=9), INVALID), (dict(x=mat(rows=2), stride=0), INVALID), (dict(x=mat(rows=2), stride=-9), INVALID),
])
def test_products_refuse(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(src=None), INVALID), (dict(src=P + 2), INVALID), (dict(dtype=2), INVALID), (dict(dtype=1, src=P + 1), INVALID),
    (dict(out=mat(rows=-1)), INVALID), (dict(out=mat(cols=0)), SHAPE), (dict(out=mat(codes=P + 16)), INVALID),
])
def test_quantize_refuses(kw, status):
    assert quantize(**kw) == status
    if "out" not in kw:
        k = {"src": P, "dtype": 0, **kw}
        assert linear(src=k["src"], src_dtype=k["dtype"]) == status


def test_linear_refuses_to_write_over_the_weights():
    assert linear(w=mat(rows=10)) == INVALID and linear(w=mat(rows=10, codes=2 * P)) == INVALID


def linear_over(src, y, stride_x, stride_y, rows=4, src_dtype=0, dtype=0):
    """x of 256 columns at src, y of 10 at y; strides in elements. The weights are far away."""
    return aw.lib.awsrc_fp8_linear(src, src_dtype, stride_x, ct.byref(mat(rows=rows, codes=P << 4, exps=P << 5)),
                                   ct.byref(mat(rows=10, codes=P << 6, exps=P << 7)), y, dtype, stride_y, P << 8, 1 << 30, None)


@pytest.mark.parametrize("kw", [
    dict(src=P, y=P, stride_x=256, stride_y=256), dict(src=P, y=P, stride_x=256, stride_y=10, rows=1),
    dict(src=P, y=P + 4 * 255, stride_x=300, stride_y=300), dict(src=P + 36, y=P, stride_x=300, stride_y=300),
    dict(src=P, y=P + 4 * (300 * 2 + 255), stride_x=300, stride_y=300),   # two rows further down
    dict(src=P + 4 * 295, y=P, stride_x=300, stride_y=300),               # y's rows against the ends of x's
    dict(src=P, y=P + 2 * 200, stride_x=300, stride_y=150, src_dtype=1),  # bf16 and float32, the same bytes a row
    dict(src=P, y=P + 4 * 300, stride_x=300, stride_y=12),                # steps that differ
    dict(src=P, y=P + 4 * 100, stride_x=0, stride_y=300),                 # one row for all of x
])
def test_linear_refuses_to_write_over_x(kw):
    assert linear_over(**kw) == INVALID


def test_matrix_bytes_are_host_only():
    def need(rows, cols):
        c, e = ct.c_size_t(), ct.c_size_t()
        return aw.lib.awsrc_fp8_matrix_bytes(rows, cols, ct.byref(c), ct.byref(e)), c.value, e.value

    assert need(1, 1) == (OK, 8 * 128, 512)
    assert need(128, 512) == (OK, 128 * 512, 512)
    assert need(129, 513) == (OK, 136 * 5 * 128, 4 * 512)
    assert need(1 << 30, 1 << 20)[:2] == (OK, 1 << 50)
    assert need(0, 5) == (OK, 0, 0) and need(-1, 5)[0] == INVALID and need(5, 0)[0] == SHAPE
    n = ct.c_size_t()
    assert aw.lib.awsrc_step_workspace_bytes(ct.byref(n)) == OK and n.value >= 256
    assert aw.lib.awsrc_step_workspace_bytes(None) == INVALID
    assert aw.lib.awsrc_step_workspace_init(None, n.value, None) == WORKSPACE
    assert aw.lib.awsrc_step_workspace_init(P, n.value - 1, None) == WORKSPACE
    assert aw.lib.awsrc_step_workspace_init(P + 16, n.value, None) == INVALID


# ----------------------------------------------------------- the binding --
def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def cpu_pool(n=2):
    return aw.awsrc_kv_pool(ints(n, 4), ints(n), ints(8), ints(1), 64)


@pytest.mark.parametrize("args,exc,msg", [
    ((ints(2, 4), ints(2, 1), ints(8), ints(1), 64), ValueError, "kv_len must be 1-D"),
    ((ints(3, 4), ints(2), ints(8), ints(1), 64), ValueError, "page_table has shape"),
    ((ints(2, 0), ints(2), ints(8), ints(1), 64), ValueError, "page_table has shape"),
    ((ints(4, 2).T, ints(2), ints(8), ints(1), 64), ValueError, "page_table must be contiguous"),
    ((ints(2, 4).long(), ints(2), ints(8), ints(1), 64), TypeError, "page_table must be"),
    ((ints(2, 4), ints(2).float(), ints(8), ints(1), 64), TypeError, "kv_len must be"),
    ((ints(2, 4), ints(2), ints(0), ints(1), 64), ValueError, "free_pages has shape"),
    ((ints(2, 4), ints(2), ints(8), ints(2), 64), ValueError, "free_count has shape"),
    ((ints(2, 4), ints(2), ints(8), ints(1), 48), ValueError, "page 48"),
])
def test_pool_tensors_are_checked(args, exc, msg):
    with pytest.raises(exc, match=msg):
        aw.awsrc_kv_pool(*args)


WS = torch.zeros(1024, dtype=torch.uint8)


@pytest.mark.parametrize("kw,exc,msg", [
    (dict(pool=7), TypeError, "awsrc_kv_pool"), (dict(n_tok=None), ValueError, "n_tok is needed"),
    (dict(n_tok=-1), ValueError, "negative"), (dict(keep=ints(3)), ValueError, "keep has shape"),
    (dict(add=ints(2).long()), TypeError, "add must be"), (dict(tok_seq=ints(4)), ValueError, "tok_seq has shape"),
    (dict(tok_slot=ints(5)), TypeError, "tok_slot must be"), (dict(workspace=WS.float()), TypeError, "workspace must be"),
    (dict(), ValueError, "a CUDA device is needed"),
])
def test_plan_arguments_are_checked(kw, exc, msg):
    a = dict(pool=cpu_pool(), keep=None, add=ints(2), workspace=WS, n_tok=5)
    a.update(kw)
    with pytest.raises(exc, match=msg):
        aw.awsrc_kv_plan(a.pop("pool"), a.pop("keep"), a.pop("add"), a.pop("workspace"), **a)


@pytest.mark.parametrize("kw,exc,msg", [
    (dict(row_start=ints(0)), ValueError, "row_start has shape"), (dict(row_start=ints(3).long()), TypeError, "row_start must be"),
    (dict(target=torch.zeros(5)), ValueError, "target must be"), (dict(target=torch.zeros(5, 9).half()), TypeError, "target must be"),
    (dict(target=torch.zeros(9, 5).T), ValueError, "last stride"), (dict(draft=torch.zeros(5, 8)), ValueError, "draft has shape"),
    (dict(ids=ints(4)), ValueError, "ids has shape"), (dict(u=torch.zeros(4)), ValueError, "u has shape"),
    (dict(r=torch.zeros(2).double()), TypeError, "r must be"), (dict(max_draft=None), ValueError, "max_draft"),
    (dict(max_draft=-1), ValueError, "max_draft"), (dict(tokens=ints(2)), ValueError, "tokens has shape"),
    (dict(keep=ints(2)), ValueError, "keep needs kv_len"), (dict(), ValueError, "a CUDA device is needed"),
])
def test_verification_arguments_are_checked(kw, exc, msg):
    a = dict(row_start=ints(3), ids=ints(5), target=torch.zeros(5, 9), draft=None, u=torch.zeros(5), r=torch.zeros(2), workspace=WS,
             max_draft=2)
    a.update(kw)
    with pytest.raises(exc, match=msg):
        aw.awsrc_verify_drafts(**a)


def test_lengths_past_31_bits_are_refused():
    """The library takes 32-bit lengths: none may arrive there cut off."""
    big = 1 << 32
    with pytest.raises(ValueError, match="n_tok"):
        aw.awsrc_kv_plan(cpu_pool(), None, ints(2), WS, n_tok=big + 5)
    a = dict(row_start=ints(3), draft=None, u=torch.zeros(5), r=torch.zeros(2), workspace=WS)
    with pytest.raises(ValueError, match="rows"):
        aw.awsrc_verify_drafts(ids=ints(5), target=torch.zeros(1, 9).expand(big + 5, 9), max_draft=2, **a)
    with pytest.raises(ValueError, match="max_draft"):
        aw.awsrc_verify_drafts(ids=ints(5), target=torch.zeros(5, 9), max_draft=big + 2, **a)
    meta = dict(dtype=torch.int32, device="meta")
    with pytest.raises(ValueError, match="vocab"):
        aw.awsrc_verify_drafts(torch.empty(3, **meta), torch.empty(5, **meta), torch.empty(5, big + 9, device="meta"), None,
                               a["u"], a["r"], WS, max_draft=2)
    with pytest.raises(ValueError, match="entries"):
        aw.awsrc_kv_pool(torch.empty(2, 4, **meta), torch.empty(2, **meta), torch.empty(big + 8, **meta), torch.empty(1, **meta), 64)


@pytest.mark.parametrize("make,exc,msg", [
    (lambda: aw.awsrc_fp8_matrix(3, 0, "cpu"), ValueError, "cannot be held"),
    (lambda: aw.awsrc_fp8_matrix(-1, 5, "cpu"), ValueError, "cannot be held"),
    (lambda: aw.Fp8Matrix(3, 5, aw.awsrc_fp8_matrix(9, 5, "cpu").codes, aw.awsrc_fp8_matrix(3, 5, "cpu").exps), ValueError, "codes has"),
    (lambda: aw.awsrc_fp8_quantize(torch.zeros(3)), ValueError, "2-D"),
    (lambda: aw.awsrc_fp8_quantize(torch.zeros(3, 4).half()), TypeError, "float32 or bfloat16"),
    (lambda: aw.awsrc_fp8_quantize(torch.zeros(4, 3).T), ValueError, "last stride"),
    (lambda: aw.awsrc_fp8_quantize(torch.zeros(3, 4)), ValueError, "a CUDA device is needed"),
    (lambda: aw.awsrc_fp8_gemm(torch.zeros(3, 4), aw.awsrc_fp8_matrix(5, 4, "cpu"), WS), TypeError, "x must come from"),
    (lambda: aw.awsrc_fp8_gemm(aw.awsrc_fp8_matrix(3, 4, "cpu"), aw.awsrc_fp8_matrix(5, 4, "cpu"), WS), ValueError, "a CUDA device"),
    (lambda: aw.awsrc_fp8_linear(torch.zeros(3, 4), aw.awsrc_fp8_matrix(5, 4, "cpu"), aw.awsrc_fp8_matrix(2, 4, "cpu"), WS), ValueError,
     "x8 is 2 x 4"),
    (lambda: _step._product(3, 4, aw.awsrc_fp8_matrix(5, 6, "cpu"), None, torch.float32, torch.device("cpu")), ValueError, "4 columns, w 6"),
    (lambda: _step._product(3, 4, aw.awsrc_fp8_matrix(5, 4, "cpu"), torch.zeros(3, 6), None, torch.device("cpu")), ValueError,
     "out has shape"),
])
def test_matrix_arguments_are_checked(make, exc, msg):
    with pytest.raises(exc, match=msg):
        make()


def test_values_of_a_matrix_read_the_layout():
    """One element at a time against the header's places."""
    gen = torch.Generator().manual_seed(0)
    m = aw.awsrc_fp8_matrix(137, 700, "cpu")
    raw, exps = m.codes.view(torch.uint8), m.exps
    for _ in range(60):
        r, k = int(torch.randint(137, (1,), generator=gen)), int(torch.randint(700, (1,), generator=gen))
        raw.zero_()
        exps.fill_(127)
        raw[k // 128, r, 16 * ((k % 128 // 16) ^ (r % 8)) + k % 16] = 0x38  # 1.0
        exps[k // 512, r // 128, r % 32, r % 128 // 32, k // 128 % 4] = 130
        v = m.values()
        assert v.shape == (137, 700) and v[r, k] == 8.0 and v.count_nonzero() == 1
