"""GPU parity of the matrices held in 8 bits: awsrc_fp8_quantize bit for bit with the
header's recipe, products exact where every sum is representable and within derived
bounds of 64 bits elsewhere."""
import math

import pytest
import torch

import step_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def aw():
    import paper_2608_23144_gb300 as aw
    assert torch.cuda.is_available()
    return aw


def assert_codes(m, codes, exps):
    c, e = ref.place(codes, exps)
    got = m.codes.cpu().double()
    rows = codes.shape[0]
    assert torch.equal(torch.isnan(got[:, :rows]), torch.isnan(c[:, :rows]))
    assert torch.equal(got[:, :rows].nan_to_num(1e9), c[:, :rows].nan_to_num(1e9))
    assert torch.equal(m.exps.cpu(), e)


def spread(rows, cols, gen):
    """Rows and blocks of very different size, single large elements, exact powers and ties among them."""
    x = torch.randn(rows, cols, generator=gen) * torch.exp2(torch.randint(-12, 13, (rows, 1), generator=gen).float())
    x[:, ::37] *= 64.0
    x[::3, ::5] = (x[::3, ::5] * 16).round() / 16
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (3, 127, 0), (8, 129, 3), (9, 512, 4), (130, 513, 0),
                                           (257, 1000, 8), (5, 2048, 1), (33, 640, 2)])
def test_quantize_follows_the_recipe(aw, dtype, rows, cols, pad):
    gen = torch.Generator().manual_seed(rows * 7 + cols)
    x = spread(rows, cols + pad, gen).to(dtype)[:, pad // 2:pad // 2 + cols]
    m = aw.awsrc_fp8_quantize(x.cuda())
    codes, exps = ref.quantize(x.double())
    assert_codes(m, codes, exps)
    assert torch.equal(m.values().cpu().double(),
                       codes * torch.ldexp(torch.ones((), dtype=torch.float64), exps).repeat_interleave(128, 1)[:, :cols])


def test_quantize_extremes(aw):
    x = torch.zeros(11, 300)
    x[0, 0] = 448.0
    x[1, 0] = 448.0 * (1 + 2.0 ** -23)
    x[2, 5] = 3.4e38
    x[3, 7] = 1e-45
    x[4, 9] = 448 * 2.0 ** -64
    x[5, 9] = 449 * 2.0 ** -64
    x[6, 130] = math.inf
    x[7, 299] = math.nan
    x[8, 10] = -math.inf
    x[9, 3] = -448.0 * 2.0 ** 100
    x[:, 64] = 2.0 ** -70
    m = aw.awsrc_fp8_quantize(x.cuda())
    assert_codes(m, *ref.quantize(x.double()))


def test_quantize_leaves_the_rows_behind_as_they_were(aw):
    m = aw.awsrc_fp8_matrix(13, 200)
    m.codes.view(torch.uint8).fill_(0x55)
    m.exps.fill_(0x77)
    aw.awsrc_fp8_quantize(torch.randn(13, 200).cuda(), out=m)
    assert (m.codes.view(torch.uint8)[:, 13:] == 0x55).all()
    assert (m.codes.view(torch.uint8)[1, :13].reshape(13, 128).sum(1) >= 0).all()
    assert (m.exps.permute(1, 3, 2, 0, 4).reshape(128, -1)[13:] == 0x77).all()
    assert torch.isfinite(m.values()).all()


def int_matrix(rows, cols, gen, lo=-3, hi=3):
    """Small whole numbers times one power of two per row: every product and sum of up to 2^18 of them is exact in binary32."""
    x = torch.randint(lo, hi + 1, (rows, cols), generator=gen).float()
    return x, torch.exp2(torch.randint(-3, 4, (rows, 1), generator=gen).float())


SIZES = [(1, 1, 1), (1, 128, 128), (1, 2048, 300), (2, 130, 129), (7, 77, 5), (16, 512, 256), (17, 640, 129), (40, 3584, 512),
         (63, 1000, 130), (64, 256, 1100), (65, 4224, 127), (128, 128, 128), (129, 300, 257), (200, 2176, 640),
         (256, 512, 384), (257, 129, 1000), (333, 5000, 177), (513, 900, 2100), (1024, 640, 1024), (2500, 520, 600)]


# many tiles for each thread block, one block of columns in a tile, long sums, shares of columns in every number, 16 rows whose
# codes do not fit beside the stages
SIZES += [(3, 256, 40000), (33, 384, 25000), (5, 100, 40000), (300, 100, 40000), (130, 4224, 12000), (16, 30000, 300), (9, 70000, 64),
          (16, 8320, 2000), (1, 640, 5000), (64, 11008, 2048), (48, 6400, 700), (100, 1280, 9000), (1, 40000, 8)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_products_of_whole_numbers_are_exact(aw, dtype, m, k, n):
    """Rows, columns and depths around every tile's edge: all sums are whole numbers below 2^24 times a power of two, so the
    tensor cores' sums are exact and any misplaced element shows."""
    gen = torch.Generator().manual_seed(m * 31 + k + n)
    x, xs = int_matrix(m, k, gen)
    w, wss = int_matrix(n, k, gen)
    want = ((x.double().cuda() @ w.double().cuda().T) * xs.double().cuda() * wss.double().cuda().T).cpu()
    assert k * 9 < 2 ** 24
    ws = aw.awsrc_step_workspace()
    xq, wq = aw.awsrc_fp8_quantize((x * xs).cuda()), aw.awsrc_fp8_quantize((w * wss).cuda())
    out = torch.full((m, n + 5), -7.0, dtype=dtype, device="cuda")
    y = aw.awsrc_fp8_gemm(xq, wq, ws, out=out[:, 2:n + 2])
    assert torch.equal(y.cpu(), want.to(dtype))
    assert (out[:, :2] == -7).all() and (out[:, n + 2:] == -7).all()
    assert aw.awsrc_workspace_status(ws) == 0


@pytest.mark.parametrize("m,k,n", [(1, 1024, 256), (33, 1152, 384), (300, 700, 300), (260, 2560, 260)])
def test_block_scales_reach_their_blocks(aw, m, k, n):
    """One nonzero block per row of x, of another scale in each row: every block's scales on both sides are told apart."""
    gen = torch.Generator().manual_seed(k)
    blocks = -(-k // 128)
    x, _ = int_matrix(m, k, gen)
    w, _ = int_matrix(n, k, gen)
    keep = torch.arange(m) % blocks
    x *= (torch.arange(k)[None] // 128 == keep[:, None])
    ex = torch.randint(-20, 20, (m, blocks), generator=gen)
    ew = torch.randint(-20, 20, (n, blocks), generator=gen)
    x *= torch.exp2(ex.float()).repeat_interleave(128, 1)[:, :k]
    w *= torch.exp2(ew.float()).repeat_interleave(128, 1)[:, :k]
    want = x.double() @ w.double().T
    y = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x.cuda()), aw.awsrc_fp8_quantize(w.cuda()), aw.awsrc_step_workspace())
    assert torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,k,n", [(1, 2048, 1100), (5, 11008, 256), (40, 3584, 1300), (100, 18944, 300), (333, 5000, 777),
                                   (700, 2100, 900)])
def test_products_against_64_bits(aw, dtype, m, k, n):
    """A sum taken over at most 2048 columns in the tensor cores has 64 steps of 32 columns, each cut off below 2^-23 of a
    running sum S_i; over random signs |S_i| grows like sqrt(i), so the error is at most 2^-23 sum_i |S_i| <= 2/3 64 2^-23 =
    5.1e-6 of the result's size, and joining the at most 10 such sums of a row rounds by 2^-24 each: 1e-5 in the norm. bf16
    sums run over all k / 32 steps, and the result is rounded once: half a step, 2^-8 relative at worst."""
    gen = torch.Generator().manual_seed(m + k)
    x = spread(m, k, gen).to(dtype).cuda()
    w = (torch.randn(n, k, generator=gen) * k ** -0.5).cuda()
    ws = aw.awsrc_step_workspace()
    wq = aw.awsrc_fp8_quantize(w)
    x8 = aw.awsrc_fp8_matrix(m, k)
    y = aw.awsrc_fp8_linear(x, wq, x8, ws)
    assert y.dtype is dtype
    assert torch.equal(y, aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), wq, ws, out_dtype=dtype))
    want = x8.values().double() @ wq.values().double().T
    err = (y.double() - want).norm() / want.norm()
    assert err <= (1e-5 if dtype is F32 else 2.0 ** -8 + 2 / 3 * k / 32 * 2.0 ** -23), float(err)
    # row by row, so that small rows count
    rows = (y.double() - want).norm(dim=1) / want.norm(dim=1)
    assert rows.max() <= (2e-5 if dtype is F32 else 2.0 ** -8 + k / 32 * 2.0 ** -23), float(rows.max())


def test_non_finite_blocks_touch_their_row_alone(aw):
    x = torch.randn(20, 400)
    w = torch.randn(150, 400)
    x[3, 200] = math.inf
    w[140, 5] = math.nan
    y = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x.cuda()), aw.awsrc_fp8_quantize(w.cuda()), aw.awsrc_step_workspace()).cpu()
    bad = torch.zeros(20, 150, dtype=torch.bool)
    bad[3], bad[:, 140] = True, True
    assert torch.equal(torch.isnan(y), bad) and torch.isfinite(y[~bad]).all()


def test_rows_behind_the_last_may_hold_anything(aw):
    """Codes and scales of the padding rows are e4m3's and the scales' NaN."""
    x, w = torch.randn(13, 300).cuda(), torch.randn(141, 300).cuda()
    ws = aw.awsrc_step_workspace()
    want = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), aw.awsrc_fp8_quantize(w), ws)
    ms = [aw.awsrc_fp8_matrix(13, 300), aw.awsrc_fp8_matrix(141, 300)]
    for m, t in zip(ms, (x, w)):
        m.codes.view(torch.uint8).fill_(0x7F)
        m.exps.fill_(255)
        aw.awsrc_fp8_quantize(t, out=m)
    assert torch.equal(aw.awsrc_fp8_gemm(ms[0], ms[1], ws), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,k,n,pad", [(1, 2048, 300, 0), (7, 1000, 5000, 3), (16, 515, 129, 1), (13, 3000, 700, 8), (31, 700, 300, 2),
                                       (64, 2048, 512, 5), (90, 640, 300, 4), (16, 30000, 200, 0)])
def test_linear_is_quantize_and_gemm(aw, dtype, m, k, n, pad):
    """Bit for bit, and x8 holds what awsrc_fp8_quantize gives, whether or not the product quantises the rows itself; a block that
    is not finite among them."""
    gen = torch.Generator().manual_seed(m * k)
    x = spread(m, k + pad, gen).to(dtype)
    x[m // 2, k // 2] = math.nan
    x = x.cuda()[:, :k]
    w = aw.awsrc_fp8_quantize(torch.randn(n, k, generator=gen).cuda())
    ws, x8, want8 = aw.awsrc_step_workspace(), aw.awsrc_fp8_matrix(m, k), aw.awsrc_fp8_quantize(x)
    y = aw.awsrc_fp8_linear(x, w, x8, ws)
    want = aw.awsrc_fp8_gemm(want8, w, ws, out_dtype=dtype)
    assert torch.equal(x8.codes.view(torch.uint8), want8.codes.view(torch.uint8)) and torch.equal(x8.exps, want8.exps)
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.nan_to_num(), want.nan_to_num())
    assert y[m // 2].isnan().all() and (m == 1 or y[(m // 2 + 1) % m].isfinite().all())
    again = aw.awsrc_fp8_linear(x, w, x8, ws)
    assert torch.equal(again.nan_to_num(), y.nan_to_num())
    stale = torch.full_like(y, 3.0).t().contiguous().t() if m > 1 and n > 1 else None
    if stale is not None:  # columns apart: refused
        with pytest.raises(ValueError):
            aw.awsrc_fp8_linear(x, w, x8, ws, out=stale)


def test_products_on_two_streams_at_once(aw):
    """Each with its own workspace and codes; both kernels need tensor memory."""
    gen = torch.Generator().manual_seed(2)
    w = aw.awsrc_fp8_quantize(torch.randn(3000, 2000, generator=gen).cuda())
    xs = [torch.randn(m, 2000, generator=gen).cuda() for m in (5, 300)]
    want = [aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), w, aw.awsrc_step_workspace()) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    sets = [(aw.awsrc_fp8_matrix(x.shape[0], 2000), aw.awsrc_step_workspace(), torch.empty_like(y)) for x, y in zip(xs, want)]
    torch.cuda.synchronize()
    for _ in range(50):
        for x, (x8, ws, y), s in zip(xs, sets, streams):
            aw.awsrc_fp8_linear(x, w, x8, ws, out=y, stream=s)
    torch.cuda.synchronize()
    for (x8, ws, y), v in zip(sets, want):
        assert torch.equal(y, v) and aw.awsrc_workspace_status(ws) == 0


def test_weights_made_just_before_the_product(aw):
    """The product's early copies of w come after the kernel that wrote it: new weights before every call, no waiting between."""
    gen = torch.Generator().manual_seed(6)
    ws = aw.awsrc_step_workspace()
    for m in (3, 40, 200):
        x = torch.randn(m, 1500, generator=gen).cuda()
        raw = [torch.randn(2500, 1500, generator=gen).cuda() for _ in range(4)]
        want = [aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(x), aw.awsrc_fp8_quantize(r), ws) for r in raw]
        torch.cuda.synchronize()
        w, x8 = aw.awsrc_fp8_matrix(2500, 1500), aw.awsrc_fp8_matrix(m, 1500)
        ys = []
        for r in raw * 5:
            aw.awsrc_fp8_quantize(r, out=w)
            ys.append(aw.awsrc_fp8_linear(x, w, x8, ws))
        torch.cuda.synchronize()
        for i, y in enumerate(ys):
            assert torch.equal(y, want[i % 4]), (m, i)


def test_empty_products(aw):
    ws = aw.awsrc_step_workspace()
    w = aw.awsrc_fp8_quantize(torch.randn(10, 64).cuda())
    none = aw.awsrc_fp8_quantize(torch.empty(0, 64, device="cuda"))
    assert aw.awsrc_fp8_gemm(none, w, ws).shape == (0, 10)
    assert aw.awsrc_fp8_gemm(w, none, ws).shape == (10, 0)
    assert aw.awsrc_fp8_linear(torch.empty(0, 64, device="cuda"), w, none, ws).shape == (0, 10)
    assert none.values().shape == (0, 64)


def test_waits_that_run_out_are_reported(aw):
    """Copies stop after 3 blocks: the products' wait runs out, the call ends and reports it, the next one is right."""
    x, w = torch.randn(300, 1024).cuda(), torch.randn(300, 1024).cuda()
    xq, wq, ws = aw.awsrc_fp8_quantize(x), aw.awsrc_fp8_quantize(w), aw.awsrc_step_workspace()
    for rows in (1, 300):
        part = aw.awsrc_fp8_quantize(x[:rows])
        for dtype in (F32, BF16):
            want = aw.awsrc_fp8_gemm(part, wq, ws, out_dtype=dtype)
            aw.awsrc_set_wait_test(2_000_000, 3)
            try:
                aw.awsrc_fp8_gemm(part, wq, ws, out_dtype=dtype)
                torch.cuda.synchronize()
            finally:
                aw.awsrc_set_wait_test()
            assert aw.awsrc_workspace_status(ws) == 4
            assert torch.equal(aw.awsrc_fp8_gemm(part, wq, ws, out_dtype=dtype), want)
            assert aw.awsrc_workspace_status(ws) == 0
    assert xq.rows == 300


def test_linear_in_a_graph_on_another_stream(aw):
    gen = torch.Generator().manual_seed(5)
    w = aw.awsrc_fp8_quantize(torch.randn(500, 700, generator=gen).cuda())
    x = torch.zeros(30, 700, device="cuda")
    x8, ws, y = aw.awsrc_fp8_matrix(30, 700), aw.awsrc_step_workspace(), torch.empty(30, 500, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        aw.awsrc_fp8_linear(x, w, x8, ws, out=y)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                aw.awsrc_fp8_linear(x, w, x8, ws, out=y)
    torch.cuda.synchronize()
    for _ in range(3):
        new = torch.randn(30, 700, generator=gen)
        x.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        want = aw.awsrc_fp8_gemm(aw.awsrc_fp8_quantize(new.cuda()), w, ws)
        assert torch.equal(y, want)


@pytest.mark.parametrize("m", [1, 7, 40, 100])
def test_linear_between_columns_of_one_matrix(aw, m):
    """x and y as columns of one buffer are a right call; y over x is none, whatever the rows."""
    gen = torch.Generator().manual_seed(m)
    k, n = 512, 256
    buf = torch.randn(m, k + n, generator=gen).cuda()
    w = aw.awsrc_fp8_quantize(torch.randn(n, k, generator=gen).cuda())
    x8, ws = aw.awsrc_fp8_matrix(m, k), aw.awsrc_step_workspace()
    x = buf[:, :k].clone()
    want = aw.awsrc_fp8_linear(x, w, x8, ws)
    aw.awsrc_fp8_linear(buf[:, :k], w, x8, ws, out=buf[:, k:])
    assert torch.equal(buf[:, k:], want) and torch.equal(buf[:, :k], x)
    for out in (buf[:, :n], buf[:, k - 1:k - 1 + n]):
        with pytest.raises(aw.AwsrcError):
            aw.awsrc_fp8_linear(buf[:, :k], w, x8, ws, out=out)
    assert torch.equal(buf[:, k:], want) and torch.equal(buf[:, :k], x)


@pytest.mark.parametrize("m", [1, 40, 100])
def test_linear_leaves_codes_where_w_has_no_rows(aw, m):
    x = torch.randn(m, 300, generator=torch.Generator().manual_seed(m)).cuda()
    x8, want = aw.awsrc_fp8_matrix(m, 300), aw.awsrc_fp8_quantize(x)
    y = aw.awsrc_fp8_linear(x, aw.awsrc_fp8_matrix(0, 300), x8, aw.awsrc_step_workspace())
    assert y.shape == (m, 0) and torch.equal(x8.values(), want.values()) and bool(x8.values().any())
