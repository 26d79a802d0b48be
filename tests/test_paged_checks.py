"""What the paged-cache calls refuse before any launch, at the C boundary (status
codes) and in the Python binding (exceptions). No GPU: pointers are made-up
numbers, tensors live on the CPU, and every call must stop at a check."""
import ctypes as ct

import pytest
import torch

import paper_2608_23144_gb300 as aw
from paper_2608_23144_gb300 import _paged

OK, INVALID, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 6  # awsrc_status

P = 1 << 20  # an aligned address that nothing reads


def cache(**over):
    c = dict(n_pages=8, page=64, n_kv_heads=2, head_dim=128, k=P, v=P, k_exp=P, v_exp=P)
    c.update(over)
    return _paged._Cache(**c)


def batch(**over):
    b = dict(n_seq=2, n_tok=5, max_new=3, max_kv=100, table_stride=4, pad_=0, q_start=P, kv_len=P, page_table=P)
    b.update(over)
    return _paged._Batch(**b)


def rows(**over):
    r = dict(p=P, tok_stride=512, head_stride=128, dtype=1, pad_=0)
    r.update(over)
    return _paged._Rows(**r)


def need(c=None, heads=4):
    n = ct.c_size_t()
    st = aw.lib.awsrc_attention_workspace_bytes(ct.byref(c or cache()), heads, ct.byref(n))
    return st, n.value


def append(c=None, b=None, heads=4, q=None, k=None, v=None, qo=None, cos=P, sin=P, rope_rows=100, rotary=128, inter=0,
           ws=P, ws_bytes=1 << 40):
    ref = [ct.byref(x or d()) for x, d in ((c, cache), (b, batch), (q, rows), (k, rows), (v, rows), (qo, rows))]
    return aw.lib.awsrc_kv_append(ref[0], ref[1], heads, ref[2], ref[3], ref[4], ref[5], cos, sin, rope_rows, rotary,
                                  inter, ws, ws_bytes, None)


def attend(c=None, b=None, heads=4, q=None, out=None, lse=None, scale=0.1, causal=1, ws=P, ws_bytes=1 << 40):
    ref = [ct.byref(x or d()) for x, d in ((c, cache), (b, batch), (q, rows), (out, rows))]
    return aw.lib.awsrc_paged_attention(ref[0], ref[1], heads, ref[2], ref[3], lse, scale, causal, ws, ws_bytes, None)


EMPTY = batch(n_tok=0)  # the one call that passes every check and launches nothing


def test_calls_without_tokens_pass():
    assert append(b=EMPTY) == OK and attend(b=EMPTY) == OK
    assert append(b=batch(n_seq=0)) == OK and attend(b=batch(n_seq=0)) == OK
    assert append(b=EMPTY, cos=None, sin=None, rope_rows=0, rotary=0) == OK  # no rotation


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("kw,status", [
    (dict(c=cache(page=48)), SHAPE), (dict(c=cache(page=256)), SHAPE), (dict(c=cache(head_dim=96)), SHAPE),
    (dict(heads=5), SHAPE), (dict(heads=0), INVALID), (dict(heads=2 * 1025), UNSUPPORTED),
    (dict(c=cache(n_pages=0)), INVALID), (dict(c=cache(n_kv_heads=0)), INVALID), (dict(c=cache(k=None)), INVALID),
    (dict(c=cache(v_exp=None)), INVALID), (dict(c=cache(k=P + 8)), INVALID), (dict(c=cache(v=P + 1)), INVALID),
    (dict(b=batch(n_seq=-1)), INVALID), (dict(b=batch(n_tok=-1)), INVALID), (dict(b=batch(max_new=-1)), INVALID),
    (dict(b=batch(max_kv=-1)), INVALID), (dict(b=batch(table_stride=0)), INVALID), (dict(b=batch(q_start=None)), INVALID),
    (dict(b=batch(kv_len=P + 2)), INVALID), (dict(b=batch(page_table=None)), INVALID),
    (dict(b=batch(table_stride=(1 << 24) + 1)), UNSUPPORTED), (dict(b=batch(n_tok=1 << 30)), UNSUPPORTED),
    (dict(q=rows(dtype=2)), INVALID), (dict(q=rows(p=None)), INVALID), (dict(q=rows(p=P + 1)), INVALID),
    (dict(q=rows(dtype=0)), INVALID),  # the other rows are bf16
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE), (dict(ws=P + 16), INVALID),
])
def test_arguments_that_both_calls_refuse(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(rotary=127), SHAPE), (dict(rotary=130), SHAPE), (dict(rotary=-2), SHAPE), (dict(inter=2), INVALID),
    (dict(cos=None), INVALID), (dict(sin=None), INVALID), (dict(rope_rows=0), INVALID), (dict(cos=P + 2), INVALID),
    (dict(k=rows(dtype=0)), INVALID), (dict(v=rows(p=None)), INVALID), (dict(qo=rows(dtype=0)), INVALID),
])
def test_arguments_that_append_refuses(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(out=rows(dtype=0)), INVALID), (dict(out=rows(p=P + 1)), INVALID), (dict(lse=P + 2), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(causal=2), INVALID),
])
def test_arguments_that_attention_refuses(kw, status):
    assert attend(**kw) == status


def test_workspace_sizes_are_host_only():
    st, n = need()
    assert st == OK and n > 0
    assert need(cache(k=None, v=None, k_exp=None, v_exp=None)) == (OK, n)  # sizes need no memory yet
    assert need(heads=5)[0] == SHAPE
    assert attend(b=EMPTY, ws_bytes=n) == OK and attend(b=EMPTY, ws_bytes=n - 1) == WORKSPACE
    c = cache()
    assert aw.lib.awsrc_attention_workspace_init(ct.byref(c), 4, None, n, None) == WORKSPACE
    assert aw.lib.awsrc_attention_workspace_init(ct.byref(c), 4, P, n - 1, None) == WORKSPACE
    assert aw.lib.awsrc_attention_workspace_init(ct.byref(c), 4, P + 16, n, None) == INVALID


# ----------------------------------------------------------- the binding --
def tensors(pages=8, heads=2, dim=128, page=64):
    f8 = torch.float8_e4m3fn
    return [torch.zeros(pages, heads, dim // 16, page, 16).to(f8), torch.zeros(pages, heads, page // 16, dim, 16).to(f8),
            *(torch.zeros(pages, heads, dtype=torch.int8) for _ in range(2))]


@pytest.mark.parametrize("i,t,exc,msg", [
    (0, torch.zeros(8, 2, 8, 64, 16), TypeError, "k must be"),
    (0, tensors()[0][0], ValueError, "k must be"),
    (0, tensors(dim=96)[0], ValueError, "head_dim 96"),
    (0, tensors(page=48)[0], ValueError, "page 48"),
    (1, tensors(page=32)[1], ValueError, "v has shape"),
    (1, tensors()[1].to(torch.float16), TypeError, "v must be"),
    (2, torch.zeros(8, 2, dtype=torch.int32), TypeError, "k_exp must be"),
    (3, torch.zeros(8, 3, dtype=torch.int8), ValueError, "v_exp has shape"),
    (3, torch.zeros(2, 8, dtype=torch.int8).T, ValueError, "v_exp must be contiguous"),
    (3, torch.zeros(8, 2, dtype=torch.int8, device="meta"), ValueError, "v_exp is on"),
])
def test_cache_tensors_are_checked(i, t, exc, msg):
    ts = tensors()
    ts[i] = t
    with pytest.raises(exc, match=msg):
        aw.awsrc_kv_cache(*ts)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


@pytest.mark.parametrize("args,exc,msg", [
    ((ints(3), ints(2, 1), ints(2, 4), 1, 1, 1), ValueError, "kv_len must be 1-D"),
    ((ints(2), ints(2), ints(2, 4), 1, 1, 1), ValueError, "q_start has shape"),
    ((ints(3), ints(2), ints(3, 4), 1, 1, 1), ValueError, "page_table has shape"),
    ((ints(3), ints(2), ints(2, 0), 1, 1, 1), ValueError, "page_table has shape"),
    ((ints(3), ints(2), ints(4, 2).T, 1, 1, 1), ValueError, "contiguous"),
    ((ints(3).long(), ints(2), ints(2, 4), 1, 1, 1), TypeError, "q_start must be"),
    ((ints(3), ints(2).float(), ints(2, 4), 1, 1, 1), TypeError, "kv_len must be"),
    ((ints(3), ints(2), ints(2, 4), -1, 1, 1), ValueError, "negative"),
    ((ints(3), ints(2), ints(2, 4), 1, 1, -1), ValueError, "negative"),
])
def test_batch_tensors_are_checked(args, exc, msg):
    with pytest.raises(exc, match=msg):
        aw.awsrc_kv_batch(*args)


@pytest.mark.parametrize("q,exc,msg", [
    (torch.zeros(5, 4, 128, dtype=torch.float16), TypeError, "q must be"),
    (torch.zeros(4, 4, 128), ValueError, "q has shape"),
    (torch.zeros(5, 3, 128), ValueError, "q has shape"),
    (torch.zeros(5, 4, 64), ValueError, "q has shape"),
    (torch.zeros(5, 512), ValueError, "q has shape"),
    (torch.zeros(5, 4, 128), ValueError, "one CUDA device"),
])
def test_queries_are_checked(q, exc, msg):
    c, b = aw.awsrc_kv_cache(*tensors()), aw.awsrc_kv_batch(ints(3), ints(2), ints(2, 4), 5, 3, 100)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(exc, match=msg):
        aw.awsrc_paged_attention(c, b, q, ws)
    with pytest.raises(exc, match=msg):
        aw.awsrc_kv_append(c, b, q, q, q, None, None, ws)
    with pytest.raises(TypeError, match="awsrc_kv_cache"):
        aw.awsrc_paged_attention(tensors(), b, q, ws)


@pytest.mark.parametrize("t,exc,msg", [
    (torch.zeros(5, 4, 64), ValueError, "k has shape"), (torch.zeros(5, 4, 128).half(), TypeError, "k must be"),
    (torch.zeros(5, 128, 4).transpose(1, 2), ValueError, "dims in a row"),
    (torch.zeros(5, 4, 128, device="meta"), ValueError, "k is on"), (None, TypeError, "k must be"),
])
def test_rows_are_checked(t, exc, msg):
    with pytest.raises(exc, match=msg):
        _paged._rows(t, "k", torch.Size((5, 4, 128)), torch.float32, torch.device("cpu"))
    assert _paged._rows(torch.zeros(5, 4, 256)[..., 3:131], "k", (5, 4, 128), torch.float32, torch.device("cpu")).tok_stride == 1024
