"""GPU parity of the serving-step calls in forms beside the usual ones: other streams,
launch forms of large vocabularies, thresholds of tiny random numbers, long sums."""
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
