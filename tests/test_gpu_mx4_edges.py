"""Products of microscaled 4-bit floating point where their results are easy to get wrong: GELU of every bf16 number, dimensions that pass a launch of some kinds of tiles."""
import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def B():
    from paper_2301_12017_amd import binding
    binding.lib()
    return binding


def _zeros(B, rows, K):
    return B.mx4_quantize(torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("M,a16", [(1, False), (40, False), (300, False), (1000, False), (1, True), (40, True)])
def test_gelu_of_every_bf16_number(B, M, a16):
    """Sums of zeros and a bias that is each finite bf16 number in turn.  log2 of Phi is fitted to 3.3e-5, and its fp32 steps add 7.2e-5 at most: 7.3e-5 of the value together, and
    1e-6 for exp2 and the last two steps; then the rounding to bf16.  Values below 2^-122 may be 0."""
    y = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    y = torch.where(torch.isfinite(y), y, torch.zeros_like(y))
    W, bias = _zeros(B, 65536, 32), y.cuda()
    if a16:
        got = B.mx4_linear_a16(torch.zeros((M, 32), dtype=torch.bfloat16, device="cuda"), W, bias, B.ACT_GELU)
    else:
        got = B.mx4_linear(_zeros(B, M, 32), W, bias, B.ACT_GELU, torch.bfloat16)
    assert torch.equal(got, got[:1].expand_as(got))
    got, x = got[0].cpu().double(), y.double()
    want = torch.where(x < 0, 0.5 * x * torch.special.erfc(-x * 0.5 ** 0.5), x * torch.special.ndtr(x))
    off = (got - want).abs()
    bad = off > 7.5e-5 * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs() + 2.0 ** -122
    assert not bad.any(), (x[bad][:4], got[bad][:4], want[bad][:4])
    # half a step is 2^-8 of the value at worst and 2^-9 at best: as close counted in steps
    step = torch.exp2(torch.floor(torch.log2(want.abs().clamp(min=2.0 ** -126))) - 7)
    assert (off <= 7.5e-5 * want.abs() + step / 2 * (1 + 2.0 ** -8) + 2.0 ** -122).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M,N", [(1, 2 ** 27), (2 ** 27, 8), (2 ** 27 + 3, 16)])
def test_products_of_a_dimension_that_some_kinds_of_tiles_do_not_launch(B, M, N, dtype):
    """2^27 rows are 2^23 tiles of 16, 2^32 threads of them: another kind takes such a call.  Zeros but for some rows, of whole numbers whose sums are exact."""
    g = torch.Generator().manual_seed(3)
    rows, few, K = max(M, N), min(M, N), 32
    tall, flat = B.MX4.new(rows, K), B.mx4_quantize(torch.randint(-4, 5, (few, K), generator=g).bfloat16().cuda())
    tall.q.zero_()
    tall.scale.fill_(0x7F)
    at = torch.tensor([0, 15, 16, 255, 257, rows // 2, rows - 33, rows - 17, rows - 1])
    x = torch.randint(-4, 5, (len(at), K), generator=g).bfloat16().cuda()
    some = B.mx4_quantize(x)
    tall.q[:, at.cuda()], tall.scale[:, at.cuda()] = some.q, some.scale
    values, others = (B.mx4_dequantize(t).cpu().double() for t in (some, flat))
    if M == rows:
        got = B.mx4_linear(tall, flat, dtype=dtype)
        assert torch.equal(got[at.cuda()].cpu().double(), (values @ others.t()).to(dtype).double())
        got[at.cuda()] = 0
    else:
        for got in (B.mx4_linear(flat, tall, dtype=dtype), B.mx4_linear_a16(B.mx4_dequantize(flat, dtype), tall)):
            assert torch.equal(got[:, at.cuda()].cpu().double(), (others @ values.t()).to(dtype).double())
            got[:, at.cuda()] = 0
            assert not got.any()
    assert not got.any()
