"""Microscaled 4-bit floating point on the GPU against plain implementations in 64 bits on the CPU: quantizer, its inverse, the products.

Codes and exponents are compared bit for bit.  Products of codes, exponents in a narrow range, are whole multiples of one number whose sums fit 24 bits: fp32 sums
hold them exactly, and the results have to be the exact ones rounded once.  Other tolerances count roundings: u = 2^-24 is half a step of fp32, h
half a step of the output's type (finfo.eps / 2)."""
import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]

U = 2.0 ** -24
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


@pytest.fixture(scope="module")
def B():
    from paper_2301_12017_amd import binding
    binding.lib()
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- the definition ----------------------------------------------------------------------------------------------------------
def _quantized(x):
    """Codes [rows, K] and bytes of exponents [rows, K / 32] of x (16-bit numbers, on the CPU)."""
    x = x.double().view(x.shape[0], -1, 32)
    most = x.abs().amax(-1)
    bad = ~torch.isfinite(x).all(-1)
    e = torch.floor(torch.log2(torch.where(bad | (most == 0), 1.0, most))) - 2
    e = torch.where(most == 0, -127.0, e).clamp(min=-127)
    a = torch.where(bad[..., None], 0.0, x.abs()) * torch.exp2(-e)[..., None]
    index = torch.zeros_like(a, dtype=torch.int64)
    for i in range(7):
        middle = (GRID[i] + GRID[i + 1]) / 2
        index += (a > middle) | ((a == middle) & (i % 2 == 1))
    codes = torch.where(bad[..., None], 0, index + 8 * torch.signbit(x))
    return codes.view(x.shape[0], -1), torch.where(bad, 255, (e + 127).long())


def _planes(codes, exponents):
    """As the library lays them out: q [planes, rows, 64], scale bytes [planes, rows, 4]."""
    rows, K = codes.shape
    pad = -K % 128
    c = torch.nn.functional.pad(codes, (0, pad)).view(rows, -1, 64, 2)
    e = torch.nn.functional.pad(exponents, (0, pad // 32)).view(rows, -1, 4)
    return (c[..., 0] | c[..., 1] << 4).to(torch.uint8).transpose(0, 1), e.to(torch.uint8).transpose(0, 1)


def _numbers(codes, exponents):
    v = GRID[codes % 8] * torch.where(codes >= 8, -1.0, 1.0)
    s = torch.where(exponents == 255, float("nan"), torch.exp2(exponents.double() - 127))
    return (v.view(*exponents.shape, 32) * s[..., None]).view(codes.shape)


def _operand(B, codes, exponents):
    q, e = _planes(codes, exponents)
    return B.MX4(q.contiguous().cuda(), e.contiguous().view(torch.int32)[..., 0].contiguous().cuda(), codes.shape[1])


def _check_quantized(B, x, Q):
    want_q, want_e = _planes(*_quantized(x))
    got_e = Q.scale[..., None].contiguous().view(torch.uint8).cpu()
    assert torch.equal(got_e, want_e), (got_e != want_e).nonzero()[:4]
    got_q = Q.q.cpu()
    assert torch.equal(got_q, want_q), (got_q != want_q).nonzero()[:4]


# ---- quantizer ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 128), (2, 96), (3, 160), (5, 544), (4, 512), (33, 1056), (129, 4096), (301, 224), (8190, 512), (4097, 800)])
def test_quantize(B, rows, K, dtype):
    x = torch.randn((rows, K), generator=_gen(rows + K)) * torch.exp(2 * torch.randn((rows, K // 32), generator=_gen(K))).repeat_interleave(32, 1)
    x[:, ::37] = 0
    x = x.to(TYPES[dtype])
    _check_quantized(B, x, B.mx4_quantize(x.cuda()))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_every_number(B, dtype):
    """All 65536 patterns in a block with a largest number of their size and with larger ones: every rounding, tie, subnormal number, infinity and NaN."""
    t = TYPES[dtype]
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(t)
    blocks = torch.zeros((65536, 32), dtype=t)
    blocks[:, 3] = x
    blocks[:, 30] = -x
    other = blocks.clone()
    up = (x.double() * 2).to(t)
    other[:, 0] = torch.where(torch.isfinite(up), up, x)
    third = blocks.clone()
    third[:, 17] = torch.where(torch.isfinite(x), torch.tensor(48.0, dtype=t), x)
    rows = torch.cat([blocks, other, third], 1)
    _check_quantized(B, rows, B.mx4_quantize(rows.cuda()))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_ties_and_signs(B, dtype):
    t = TYPES[dtype]
    x = torch.zeros((1, 64), dtype=t)
    x[0, :16] = torch.tensor([4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0])
    x[0, 32:40] = torch.tensor([7.0, -7.875, 6.5, 0.125, -0.1, 5.5, 4.5, 1.0])
    Q = B.mx4_quantize(x.cuda())
    _check_quantized(B, x, Q)
    got = B.mx4_dequantize(Q, t).cpu()
    assert got[0, :16].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 0] and got[0, 32:40].tolist() == [6, -6, 6, 0, 0, 6, 4, 1]
    assert torch.signbit(got[0, [8, 15, 36]]).all() and not torch.signbit(got[0, [1, 35]]).any()


@pytest.mark.parametrize("rows,K", [(3, 96), (4100, 544)])
def test_quantize_strided_rows_and_what_lies_around(B, rows, K):
    """Columns of a wider matrix whose others are NaN, into the middle of a buffer whose rest stays."""
    wide = torch.full((rows, K + 40), float("nan"), dtype=torch.bfloat16)
    x = torch.randn((rows, K), generator=_gen(7)).bfloat16()
    wide[:, 16:16 + K] = x
    planes = -(-K // 128)
    q, s = torch.full((planes * rows * 64 + 256,), 77, dtype=torch.uint8, device="cuda"), torch.full((planes * rows + 8,), 77, dtype=torch.int32, device="cuda")
    out = B.MX4(q[128:-128].view(planes, rows, 64), s[3:-5].view(planes, rows), K)
    B.mx4_quantize(wide.cuda()[:, 16:16 + K], out)
    _check_quantized(B, x, out)
    assert (q[:128] == 77).all() and (q[-128:] == 77).all() and (s[:3] == 77).all() and (s[-5:] == 77).all()


def test_quantize_behind_two_to_the_32(B):
    rows, K = 70000, 65536
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((5, K), generator=_gen(3)).bfloat16()
    x[-5:] = tail.cuda()
    Q = B.mx4_quantize(x)
    want = B.mx4_quantize(tail.cuda())
    assert torch.equal(Q.q[:, -5:], want.q) and torch.equal(Q.scale[:, -5:], want.scale) and not Q.q[:, :-5].any() and not Q.scale[:, :-5].any()
    y = B.mx4_dequantize(Q)
    assert torch.equal(y[-5:], B.mx4_dequantize(want)) and not y[-10:-5].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_dequantize_every_number(B, dtype):
    codes = torch.arange(16).repeat(256, 2)
    exponents = torch.arange(256)[:, None]
    got = B.mx4_dequantize(_operand(B, codes, exponents), TYPES[dtype]).cpu()
    want = _numbers(codes, exponents).to(TYPES[dtype])
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(1).double(), want.nan_to_num(1).double())
    assert torch.equal(torch.signbit(got[:255]), torch.signbit(want[:255]))


@pytest.mark.parametrize("rows,K", [(1, 32), (7, 96), (18, 544), (1000, 1056)])
def test_dequantize(B, rows, K):
    codes, exponents = torch.randint(0, 16, (rows, K), generator=_gen(1)), torch.randint(110, 140, (rows, K // 32), generator=_gen(2))
    assert torch.equal(B.mx4_dequantize(_operand(B, codes, exponents)).cpu().double(), _numbers(codes, exponents))


def test_operands_as_checkpoints_hold_them(B):
    codes, exponents = torch.randint(0, 16, (9, 160), generator=_gen(1)), torch.randint(0, 255, (9, 5), generator=_gen(2))
    packed = (codes[:, ::2] | codes[:, 1::2] << 4).to(torch.uint8)
    got, want = B.MX4.from_rows(packed.cuda(), exponents.to(torch.uint8).cuda()), _operand(B, codes, exponents)
    assert got.K == 160 and torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)


def test_operands_as_checkpoints_hold_them_strided_and_none(B):
    codes, exponents = torch.randint(0, 256, (6, 192), generator=_gen(1)).to(torch.uint8).cuda(), torch.randint(0, 255, (6, 12), generator=_gen(2)).to(torch.uint8).cuda()
    want, got = B.MX4.from_rows(codes[::2, :128].contiguous(), exponents[::2, :8].contiguous()), B.MX4.from_rows(codes[::2, :128], exponents[::2, :8])
    assert torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)
    none = B.MX4.from_rows(codes[:0], exponents[:0])
    assert (none.rows, none.K) == (0, 384) and B.mx4_linear(none, B.MX4.from_rows(codes.repeat(4, 1), exponents.repeat(4, 1))).shape == (0, 24)


# ---- products ----------------------------------------------------------------------------------------------------------------
def _exact_operand(g, rows, K):
    """Numbers that are multiples of 1/2 up to 24 (exponents 0 .. 2)."""
    return torch.randint(0, 16, (rows, K), generator=g), torch.randint(127, 130, (rows, K // 32), generator=g)


SIZES = [(1, 8, 32), (1, 24, 128), (2, 264, 96), (5, 1024, 1056), (16, 136, 288), (17, 72, 512), (33, 520, 160), (48, 40, 4096), (64, 256, 256), (65, 128, 640),
         (127, 136, 384), (130, 264, 1056), (200, 1000, 512), (256, 256, 128), (257, 520, 1184), (300, 4096, 96), (515, 768, 800), (1031, 264, 2080), (2050, 1544, 288)]
# the kinds of tiles in LDS, two sizes of each: 64 x 64, 64 x 128, 128 x 128, 128 x 256, 256 x 256 (the last two with tiles taken in quarters)
TILES = [(300, 2056, 1056), (330, 2120, 1184), (257, 2056, 32), (300, 4168, 672), (1000, 4104, 288), (200, 12296, 32), (700, 8200, 160), (777, 8328, 224), (5001, 2056, 96),
         (4300, 4104, 160), (4609, 3848, 544)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES + TILES)
def test_linear_exact(B, M, N, K, dtype):
    """Products are multiples of 1/4 below 2^10: sums of up to 4096 of them fit 24 bits."""
    g, t = _gen(M + N + K), TYPES[dtype]
    a, w = _exact_operand(g, M, K), _exact_operand(g, N, K)
    want = _numbers(*a) @ _numbers(*w).t()
    got = B.mx4_linear(_operand(B, *a), _operand(B, *w), dtype=t)
    assert got.shape == (M, N) and got.dtype == t
    assert torch.equal(got.cpu(), want.float().to(t)), (got.cpu().double() - want).abs().max()


def _gelu64(y):
    return y * torch.special.ndtr(y)


def _close(got, y, size, n, t, gelu, floor=0.0):
    """n roundings of fp32 sums of this size, a unit each at most (truncation allowed), then GELU (slope at most 1.13; its own error 9e-5 of the value
    and 7e-7), then one rounding."""
    err = n * 2 * U * size + floor
    want = y
    if gelu:
        want, err = _gelu64(y), 1.13 * err + 9e-5 * _gelu64(y).abs() + 7e-7
        if t == torch.float16:                                    # (subnormal results: steps of 2^-24)
            err = err + 2.0 ** -25
    h = torch.finfo(t).eps / 2
    off = (got.double() - want).abs()
    assert (off <= err * (1 + h) + h * want.abs() + (2.0 ** -25 if t == torch.float16 else 0.0)).all(), float((off / (err + h * want.abs())).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 264, 1056), (13, 72, 544), (40, 1032, 320), (90, 264, 2080), (301, 520, 1056), (1100, 776, 256)])
def test_linear_of_quantized_rows(B, M, N, K, gelu, dtype):
    """Activations and weights as the quantizer leaves them, a bias; K additions in any order, and the bias."""
    g, t = _gen(M + K), TYPES[dtype]
    X = (torch.randn((M, K), generator=g) * torch.exp(torch.randn((M, 1), generator=g))).to(t)
    Wf, b = (torch.randn((N, K), generator=g) * 0.05).to(t), torch.randn((N,), generator=g).mul(0.1).to(t)
    a, w = _numbers(*_quantized(X)), _numbers(*_quantized(Wf))
    got = B.mx4_linear(B.mx4_quantize(X.cuda()), B.mx4_quantize(Wf.cuda()), b.cuda(), B.ACT_GELU if gelu else B.ACT_NONE, t)
    _close(got.cpu(), a @ w.t() + b.double(), a.abs() @ w.abs().t() + b.double().abs(), K + 1, t, gelu)


@pytest.mark.parametrize("M", [1, 20, 100, 300, 1100])
def test_linear_takes_every_exponent(B, M):
    """Blocks 2^-127 times blocks 2^127, and the other way round: exponents add up, whatever each of them is."""
    g, N, K = _gen(4), 264, 384
    a, w = torch.randint(0, 16, (M, K), generator=g), torch.randint(0, 16, (N, K), generator=g)
    ea, ew = torch.tensor([0, 254, 1, 253, 127, 200, 54, 127, 254, 3, 0, 251]), torch.tensor([254, 0, 253, 1, 127, 54, 200, 127, 0, 251, 254, 3])
    want = (GRID[a % 8] * torch.where(a > 7, -1.0, 1.0)) @ (GRID[w % 8] * torch.where(w > 7, -1.0, 1.0)).t()
    got = B.mx4_linear(_operand(B, a, ea.expand(M, 12).clone()), _operand(B, w, ew.expand(N, 12).clone()))
    assert torch.equal(got.cpu(), want.float().half())            # (multiples of 1/4: sums of 384 fit fp32, and are rounded once where they pass fp16's 512)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M", [3, 50, 150, 600])
def test_linear_blocks_that_are_nan(B, M, gelu, dtype):
    g, N, K = _gen(5), 136, 416
    a, w = _exact_operand(g, M, K), _exact_operand(g, N, K)
    clean = B.mx4_linear(_operand(B, *a), _operand(B, *w), None, B.ACT_GELU if gelu else B.ACT_NONE, TYPES[dtype]).cpu()
    a[1][M // 2, 7] = 255
    w[1][5, 2] = w[1][N - 1, 12] = 255
    got = B.mx4_linear(_operand(B, *a), _operand(B, *w), None, B.ACT_GELU if gelu else B.ACT_NONE, TYPES[dtype]).cpu()
    bad = torch.zeros((M, N), dtype=torch.bool)
    bad[M // 2] = bad[:, 5] = bad[:, N - 1] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", TILES)
def test_kinds_of_tiles_agree(B, M, N, K, dtype):
    """With a bias, GELU and blocks that are NaN: the bits that few rows at a time give (their sums are exact, and GELU is one function)."""
    g, t = _gen(M + K), TYPES[dtype]
    a, w = _exact_operand(g, M, K), _exact_operand(g, N, K)
    a[1][M // 2, 0] = w[1][N // 3, 0] = 255
    a[1][:, 0] = torch.where(a[1][:, 0] == 255, 255, 122)         # (smaller sums, where GELU is more than max(x, 0))
    if K > 32:
        a[1][:, 1:] = 121
    b = torch.randint(-8, 9, (N,), generator=g).to(t).cuda()
    W = _operand(B, *w)
    got = B.mx4_linear(_operand(B, *a), W, b, B.ACT_GELU, t).cpu()
    rows = sorted({0, 1, 31, 64, M // 2, M // 2 + 1, M - 66, M - 33, M - 2, M - 1})
    few = B.mx4_linear(_operand(B, a[0][rows], a[1][rows]), W, b, B.ACT_GELU, t).cpu()
    assert torch.equal(got[rows].view(torch.int16)[~few.isnan()], few.view(torch.int16)[~few.isnan()])
    assert torch.equal(got[rows].isnan(), few.isnan()) and got[M // 2].isnan().all() and got[:, N // 3].isnan().all() and got.isnan().sum() == M + N - 1


def test_linear_past_the_largest_number(B):
    """Sums past fp32 and past fp16 are infinities, GELU of them too; far below zero it is 0."""
    for M, N in ((2, 16), (70, 16), (400, 16), (300, 2056), (1000, 4104)):
        a = torch.full((M, 32), 7), torch.full((M, 1), 254)
        w = torch.full((N, 32), 7), torch.full((N, 1), 254)
        w[0][1] = 15
        got = B.mx4_linear(_operand(B, *a), _operand(B, *w), dtype=torch.bfloat16).cpu()
        assert (got[:, 0] == float("inf")).all() and (got[:, 1] == -float("inf")).all()
        for t in TYPES.values():
            got = B.mx4_linear(_operand(B, *a), _operand(B, *w), None, B.ACT_GELU, t).cpu()
            assert (got[:, 0] == float("inf")).all() and (got[:, 1] == 0).all()
        a[1][:], w[1][:] = 134, 134
        got = B.mx4_linear(_operand(B, *a), _operand(B, *w)).cpu()
        assert (got[:, 0] == float("inf")).all() and (got[:, 1] == -float("inf")).all()


@pytest.mark.parametrize("M", [1, 30, 200, 700])
def test_linear_writes_its_rows_alone(B, M):
    g, N, K = _gen(6), 72, 96
    a, w = _exact_operand(g, M, K), _exact_operand(g, N, K)
    buf = torch.full((M * N + 512,), 3.0, dtype=torch.float16, device="cuda")
    out = buf[256:-256].view(M, N)
    B.mx4_linear(_operand(B, *a), _operand(B, *w), out=out)
    assert torch.equal(out.cpu(), (_numbers(*a) @ _numbers(*w).t()).float().half()) and (buf[:256] == 3).all() and (buf[-256:] == 3).all()


def test_linear_behind_two_to_the_32(B):
    """Codes past 4 GB: the last rows of a tall operand, as activations and as weights."""
    rows, K = 140000, 65536
    Q = B.MX4.new(rows, K)
    Q.q.zero_()
    Q.scale.fill_(0x7F7F7F7F)
    g = _gen(8)
    tail, small = (torch.randint(0, 16, (24, K), generator=g), torch.full((24, K // 32), 127)), (torch.randint(0, 16, (8, K), generator=g), torch.full((8, K // 32), 120))
    T, S = _operand(B, *tail), _operand(B, *small)
    Q.q[:, -24:] = T.q
    got = B.mx4_linear(Q, S, dtype=torch.bfloat16)
    assert torch.equal(got[-24:], B.mx4_linear(T, S, dtype=torch.bfloat16)) or (got[-24:].float() - B.mx4_linear(T, S, dtype=torch.bfloat16).float()).abs().max() <= 2.0 ** -8 * got[-24:].float().abs().max()
    assert not got[:-24].any()
    got = B.mx4_linear(S, Q, dtype=torch.bfloat16)
    assert (got[:, -24:].float() - B.mx4_linear(S, T, dtype=torch.bfloat16).float()).abs().max() <= 2.0 ** -8 * got.float().abs().max() and not got[:, :-24].any()
    x = torch.randn((3, K), generator=g).bfloat16().cuda()
    got, want = B.mx4_linear_a16(x, Q)[:, -24:].float(), B.mx4_linear_a16(x, T).float()
    assert (got - want).abs().max() <= 2.0 ** -8 * want.abs().max()


# ---- products with 16-bit activations ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 8, 32), (1, 520, 96), (2, 264, 160), (5, 136, 1056), (15, 40, 544), (16, 72, 128), (17, 1032, 288), (33, 264, 4096), (48, 88, 608),
                                   (64, 520, 256), (65, 136, 384), (150, 72, 800), (7, 13000, 352), (31, 12296, 64), (60, 6200, 160),
                                   (3, 16008, 544), (13, 16024, 1056), (64, 16008, 32), (50, 24008, 160), (33, 8200, 1056)])
def test_a16_exact(B, M, N, K, dtype):
    """Whole numbers up to 31 times multiples of 1/2 up to 24: sums of 4096 products fit 24 bits."""
    g, t = _gen(M + N + K), TYPES[dtype]
    w = _exact_operand(g, N, K)
    x = torch.randint(-15, 16, (M, K), generator=g).to(t)
    wide = torch.full((M, K + 24), float("nan"), dtype=t)
    wide[:, 8:8 + K] = x
    want = x.double() @ _numbers(*w).t()
    got = B.mx4_linear_a16(wide.cuda()[:, 8:8 + K], _operand(B, *w))
    assert got.dtype == t and torch.equal(got.cpu(), want.float().to(t)), (got.cpu().double() - want).abs().max()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 264, 1056), (13, 776, 544), (29, 1032, 320), (64, 264, 2080), (90, 40, 256)])
def test_a16(B, M, N, K, gelu, dtype):
    g, t = _gen(M + K), TYPES[dtype]
    X = (torch.randn((M, K), generator=g) * torch.exp(torch.randn((M, 1), generator=g))).to(t)
    w, b = (torch.randint(0, 16, (N, K), generator=g), torch.randint(118, 126, (N, K // 32), generator=g)), torch.randn((N,), generator=g).mul(0.1).to(t)
    x, v = X.double(), _numbers(*w)
    got = B.mx4_linear_a16(X.cuda(), _operand(B, *w), b.cuda(), B.ACT_GELU if gelu else B.ACT_NONE)
    # (a block's sum, its product with the power of two exact, and the sum of blocks: K additions and the bias)
    _close(got.cpu(), x @ v.t() + b.double(), x.abs() @ v.abs().t() + b.double().abs(), K + 1, t, gelu)


def test_a16_takes_every_exponent(B):
    """Weights from 2^-128 to 2^127, which no 16-bit type holds beside each other; activations that bring them back."""
    g, M, N = _gen(4), 3, 40
    e = torch.tensor([0, 1, 20, 100, 127, 150, 230, 250])
    w = torch.randint(0, 16, (N, 256), generator=g)
    x = torch.zeros((M, 8, 32), dtype=torch.float64)
    for m in range(M):
        for i, b in enumerate(e.tolist()):
            x[m, i] = torch.randint(-4, 5, (32,), generator=g).double() * 2.0 ** max(min(127 - b, 110), -120)
    for i in range(8):                                            # one block at a time: their results are 2^100 apart
        xi = torch.zeros_like(x)
        xi[:, i] = x[:, i]
        want = xi.view(M, 256) @ _numbers(w, e.expand(N, 8)).t()
        got = B.mx4_linear_a16(xi.view(M, 256).bfloat16().cuda(), _operand(B, w, e.expand(N, 8).clone()))
        assert torch.equal(got.cpu().double(), want.to(torch.bfloat16).double()), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [4, 40])
def test_a16_infinities_and_nans_stay_in_their_rows(B, M, dtype):
    g, N, K = _gen(9), 72, 288
    w = _exact_operand(g, N, K)
    w[0][:, 100] = 3                                              # (1.5 times a power of two: an infinity times it is one)
    w[0][2, 100] = 0
    x = torch.randint(-15, 16, (M, K), generator=g).to(TYPES[dtype])
    clean = B.mx4_linear_a16(x.cuda(), _operand(B, *w)).cpu()
    x[1, 100], x[3, 7] = float("inf"), float("nan")
    w[1][6, 1] = 255
    got = B.mx4_linear_a16(x.cuda(), _operand(B, *w)).cpu()
    others = torch.ones((M, N), dtype=torch.bool)
    others[1], others[3], others[:, 6] = False, False, False
    assert torch.equal(got[others], clean[others]) and got[3].isnan().all() and got[:, 6].isnan().all() and got[1, 2].isnan()
    rest = [n for n in range(N) if n not in (2, 6)]
    assert (got[1, rest] == float("inf")).all()


# ---- as programs call them -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M", [3, 300])
def test_captured_and_replayed(B, M):
    """Quantizer and both products in a graph, replayed on other inputs, with eager work between; another stream than the default one."""
    g, N, K = _gen(11), 264, 544
    X, W = torch.randn((M, K), generator=g).half().cuda(), B.mx4_quantize(torch.randn((N, K), generator=g).half().cuda())
    quantize = B.PreparedMX4Quantize(X)
    calls = [quantize, B.PreparedMX4Linear(quantize.out, W), B.PreparedMX4LinearA16(X, W)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for call in calls:
            call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in calls:
            call()
    for i in range(4):
        X.copy_(torch.randn((M, K), generator=g).half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(calls[1].out, B.mx4_linear(B.mx4_quantize(X), W)) and torch.equal(calls[2].out, B.mx4_linear_a16(X, W))


def test_nothing_to_do(B):
    W = B.mx4_quantize(torch.randn((16, 96)).half().cuda())
    none = torch.empty((0, 96), dtype=torch.float16, device="cuda")
    A = B.mx4_quantize(none)
    assert A.q.shape == (1, 0, 64) and B.mx4_dequantize(A).shape == (0, 96) and B.mx4_linear(A, W).shape == (0, 16) and B.mx4_linear_a16(none, W).shape == (0, 16)


def test_same_bits_every_time(B):
    g, K = _gen(12), 2080
    W = B.mx4_quantize(torch.randn((520, K), generator=g).half().cuda())
    for M in (1, 40, 300, 1500):
        X = torch.randn((M, K), generator=g).half().cuda()
        A = B.mx4_quantize(X)
        first, few = B.mx4_linear(A, W), B.mx4_linear_a16(X, W)
        for _ in range(3):
            assert torch.equal(first, B.mx4_linear(A, W)) and torch.equal(few, B.mx4_linear_a16(X, W))
