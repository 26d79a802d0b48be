"""GPU parity of the 8-bit products where sums are long, waits run out in every kernel,
rows are written beside others that stay, and weights come out of the records' decoder."""
import pytest
import torch

import step_ref as ref
from test_gpu_fp8 import aw, int_matrix, spread  # noqa: F401

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def test_quantize_writes_its_rows_and_no_others(aw):  # noqa: F811
    """13 of 16 rows of codes and of 128 of scales: the first as the recipe has them, the others as they were."""
    x = spread(13, 200, torch.Generator().manual_seed(4))
    m = aw.awsrc_fp8_matrix(13, 200)
    m.codes.view(torch.uint8).fill_(0x55)
    m.exps.fill_(0x77)
    aw.awsrc_fp8_quantize(x.cuda(), out=m)
    codes, exps = ref.place(*ref.quantize(x.double()))
    assert torch.equal(m.codes.cpu()[:, :13].double(), codes[:, :13])
    assert (m.codes.view(torch.uint8)[:, 13:] == 0x55).all()
    rows = m.exps.cpu().permute(1, 3, 2, 0, 4).reshape(128, -1)
    assert torch.equal(rows[:13], exps.permute(1, 3, 2, 0, 4).reshape(128, -1)[:13]) and (rows[13:] == 0x77).all()


@pytest.mark.parametrize("m", [1, 5, 40, 70, 300])
@pytest.mark.parametrize("dtype,blocks", [(F32, 16), (BF16, 256)])
def test_sums_leave_the_tensor_cores_as_often_as_stated(aw, m, dtype, blocks):  # noqa: F811
    """A one in the first 2048 columns (bf16: 32768), small products in the second, a one taken off in the third. The
    stretches' sums are 1, 2^-23 and -1, exact, and so are their additions in binary32: the result is 2^-23 to the bit. In one
    sum without a stop the small products, 2^-29 of the one (2^-33) per 32 columns, would be cut off beside it. Rows enough
    that columns are not shared; another power of two for each row."""
    n, k = 9800, 3 * blocks * 128
    x, w = (torch.zeros(r, k, dtype=BF16, device="cuda") for r in (m, n))
    low = slice(blocks * 128, 2 * blocks * 128)
    x[:, 0], w[:, 0] = 1.0, 1.0
    x[:, low] = 2.0 ** -17
    w[:, low] = 2.0 ** -23 / (blocks * 128) * 2.0 ** 17
    x[:, 2 * blocks * 128], w[:, 2 * blocks * 128] = 1.0, -1.0
    xs, wsc = (torch.exp2((torch.arange(r, device="cuda") * 7 % 9 - 4).float()) for r in (m, n))
    x8, w8 = aw.awsrc_fp8_quantize(x * xs[:, None].to(BF16)), aw.awsrc_fp8_quantize(w * wsc[:, None].to(BF16))
    ws = aw.awsrc_step_workspace()
    y = aw.awsrc_fp8_gemm(x8, w8, ws, out_dtype=dtype)
    assert torch.equal(y.float(), 2.0 ** -23 * xs[:, None] * wsc)
    assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("m,n", [(1, 300), (5, 1000), (16, 10000), (40, 700), (64, 10000), (100, 300), (300, 1111)])
def test_long_sums_of_positive_terms(aw, m, n):  # noqa: F811
    """Where cutting off adds up. A stretch of 2048 columns is 64 steps of 32 columns, each cut off by less than a unit of
    binary32, 2^-23 of the running sum S_i at most; factors between 1/2 and 1 keep S_i within 3% of i / 64 of the whole, so
    sum_i 2^-23 S_i <= 33.5 2^-23 of it. The 14 stretches of 27648 columns (at most 8 shares of columns begin one more each) join with
    22 roundings of 2^-24 at most: 4.0e-6 + 1.4e-6, every element. Without stops 864 steps are off by 1.2e-5 (measured)."""
    gen = torch.Generator(device="cuda").manual_seed(m)
    x, w = (0.5 + 0.5 * torch.rand(r, 27648, generator=gen, device="cuda") for r in (m, n))
    x8, w8, ws = aw.awsrc_fp8_matrix(m, 27648), aw.awsrc_fp8_quantize(w), aw.awsrc_step_workspace()
    y = aw.awsrc_fp8_linear(x, w8, x8, ws)
    want = x8.values().double() @ w8.values().double().T
    off = ((y.double() - want) / want).abs().max()
    assert off <= 33.5 * 2.0 ** -23 + 22 * 2.0 ** -24, float(off)
    # bf16: one sum of 864 steps, 432.5 2^-23 at most, and a rounding of half a step
    y = aw.awsrc_fp8_gemm(x8, w8, ws, out_dtype=BF16)
    off = ((y.double() - want) / want).abs().max()
    assert off <= 2.0 ** -8 + 445 * 2.0 ** -23, float(off)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,k,n", [(100, 70000, 300), (300, 40000, 600), (65, 98400, 129)])
def test_whole_numbers_over_many_columns_by_pairs(aw, dtype, m, k, n):  # noqa: F811
    """Several stretches of 32768 columns in the pairs' kernel: sums of whole numbers below 2^24, exact."""
    gen = torch.Generator().manual_seed(k)
    (x, xs), (w, wss) = int_matrix(m, k, gen), int_matrix(n, k, gen)
    want = (x.double().cuda() @ w.double().cuda().T) * xs.double().cuda() * wss.double().cuda().T
    assert k * 9 < 2 ** 24
    ws = aw.awsrc_step_workspace()
    y = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize((x * xs).cuda()), aw.awsrc_fp8_quantize((w * wss).cuda()), ws, out_dtype=dtype)
    assert torch.equal(y, want.to(dtype)) and aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("m,n,k", [(1, 300, 1024), (7, 10000, 1024), (16, 300, 2048), (40, 300, 1024), (64, 10000, 640), (16, 200, 30000),
                                   (100, 300, 1024)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("stall", [0, 3])
def test_waits_that_run_out_in_every_kernel(aw, m, n, k, dtype, stall):  # noqa: F811
    """Copies stop after `stall` blocks, in awsrc_fp8_linear (rows quantised in the kernel, or in one before it) and
    awsrc_fp8_gemm: the waits of 2 ms run out, the call ends and reports it, the next one is right."""
    gen = torch.Generator().manual_seed(m + k)
    x = torch.randn(m, k, generator=gen).to(dtype).cuda()
    w8, ws, x8 = aw.awsrc_fp8_quantize(torch.randn(n, k, generator=gen).cuda()), aw.awsrc_step_workspace(), aw.awsrc_fp8_matrix(m, k)
    want = aw.awsrc_fp8_linear(x, w8, x8, ws)
    calls = (lambda: aw.awsrc_fp8_linear(x, w8, x8, ws), lambda: aw.awsrc_fp8_gemm(x8, w8, ws, out_dtype=dtype))
    for call in calls:
        aw.awsrc_set_wait_test(2_000_000, stall)
        try:
            call()
            torch.cuda.synchronize()
        finally:
            aw.awsrc_set_wait_test()
        assert aw.awsrc_workspace_status(ws) == 4
        assert torch.equal(call(), want) and aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_rows_are_quantised_where_that_is_shorter(aw, dtype):  # noqa: F811
    """11008 rows of w share no columns, so a thread block has all 16 blocks of a row of x: two rows of bf16 and three of float32
    are quantised in the product's kernel, more of them in one before it. The same results, with new weights written just
    before every call."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    k, n = 2048, 11008
    ws, w8 = aw.awsrc_step_workspace(), aw.awsrc_fp8_matrix(n, k)
    raw = [torch.randn(n, k, generator=gen, device="cuda") for _ in range(2)]
    kept = [aw.awsrc_fp8_quantize(r) for r in raw]
    for m in (1, 2, 3, 4, 9, 16):
        x = torch.randn(m, k, generator=gen, device="cuda").to(dtype)
        want8 = aw.awsrc_fp8_quantize(x)
        want = [aw.awsrc_fp8_gemm(want8, w, ws, out_dtype=dtype) for w in kept]
        x8, ys = aw.awsrc_fp8_matrix(m, k), []
        torch.cuda.synchronize()
        for i in range(8):
            aw.awsrc_fp8_quantize(raw[i % 2], out=w8)
            before = aw.awsrc_kernel_launches()
            ys.append(aw.awsrc_fp8_linear(x, w8, x8, ws))
            assert aw.awsrc_kernel_launches() - before == (1 if m <= (2 if dtype is BF16 else 3) else 2)
        torch.cuda.synchronize()
        assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(ys))
        assert torch.equal(x8.codes.view(torch.uint8), want8.codes.view(torch.uint8)) and torch.equal(x8.exps, want8.exps)


@pytest.mark.parametrize("m", [4, 100])
def test_products_of_decoded_weights(aw, m):  # noqa: F811
    """W_hat out of the records' decoder, held in 8 bits for the rows that the packed product does not take. A code is within half
    a step, 2^-4 of a normal value or 2^-10 2^e of a subnormal one, of what it stands for, on both sides of the product:
    dx = 2^-4 |x| + 2^(ex - 10), dw likewise, so |y - x W_hat^T| <= |x| dw + dx |w| + dx dw, and sums off by 4.0e-6 + 22 2^-24 of
    |x| |w| at most (as for positive terms). The packed product of the same records is within its own stated bound."""
    from synth import make_module
    rows, cols, gen = 512, 2048, torch.Generator().manual_seed(m)
    mod = make_module(rows, cols, seed=9, device="cuda")
    prm = aw.params(C=64, P=4, b=4, S=256)
    back = aw.awsrc_rtn_quantize(mod["W"], w0_dtype=F32)
    mod = dict(mod, W=mod["W"].float(), W0=back["W0"])
    cands = aw.awsrc_encode_tiles(prm, [mod])
    stream, counts, _ = aw.awsrc_select_records(prm, [mod], cands, [0.162])
    k = int(counts.sum())
    assert k > 100
    w = aw.awsrc_decode_apply(prm, [mod], stream, k, out_dtype=F32)[0]
    x = torch.randn(m, cols, generator=gen).cuda()
    w8, x8, ws = aw.awsrc_fp8_quantize(w), aw.awsrc_fp8_matrix(m, cols), aw.awsrc_step_workspace()
    y = aw.awsrc_fp8_linear(x, w8, x8, ws).double()

    def half(t):
        amax = t.double().abs().view(t.shape[0], -1, 128).amax(2)
        e = torch.ceil(torch.log2(amax / 448)).clamp(min=-64)
        return 2.0 ** -4 * t.double().abs() + torch.exp2(e - 10).repeat_interleave(128, 1)

    absx, absw, dx, dw = x.double().abs(), w.double().abs(), half(x), half(w)
    want = x.double() @ w.double().T
    bound = absx @ dw.T + dx @ absw.T + dx @ dw.T + (33.5 * 2.0 ** -23 + 22 * 2.0 ** -24) * ((absx + dx) @ (absw + dw).T)
    assert ((y - want).abs() <= bound).all()
    # in the mean square 2^-4 / sqrt(3) a side at most, 0.051 together; half as much again
    assert (y - want).norm() <= 0.077 * want.norm()
    if m <= 8:
        side = aw.awsrc_sidecar_prepare(prm, [(rows, cols)], stream, k)
        packed = aw.awsrc_packed_gemv(prm, [(rows, cols)], 0, back, x, sidecar=side).double()
        w0 = back["W0"].double()
        own = (cols / 32 + 32) * 2.0 ** -24 * (absx @ (w0.abs() + (w.double() - w0).abs()).T) + 2.0 ** -24 * (absx @ absw.T)
        assert ((packed - want).abs() <= own).all()
        assert ((y - packed).abs() <= bound + own).all()
