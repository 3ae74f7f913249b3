"""Products of microscaled 4-bit floating point where their results are easy to get wrong: GELU of every bf16 number."""
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
