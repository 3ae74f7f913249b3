"""Token generation on the GPU where it can go wrong: rows of NaN, infinities, scales far apart, sizes at their limits, single rows of wider
arrays, shared workspaces.  Oracles and tolerances as in test_gpu_generation.py."""
import pytest
import torch

from tests.gpu_util import has_gpu
from tests.test_gpu_generation import B, _gen, _random_cache  # noqa: F401 (B is a fixture)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n, keys, window", [(40, 40, 0), (100, 100, 0), (3, 3, 0), (40, 600, 17), (3, 600, 17), (300, 330, 0)])
def test_a_row_of_nan_stays_nan_where_its_steps_are_masked(B, n, keys, window, D):
    """Rows near the beginning of a fresh prompt, and behind a short window: no step of theirs is without a mask."""
    g = _gen(n + D)
    cache = _random_cache(B, g, 40, 2, 16, D)
    q = torch.randn((n, 4, D), generator=g).half().cuda()
    call = B.PreparedKV8Attention(q, cache, torch.arange(40, dtype=torch.int32, device="cuda")[None], torch.tensor([keys], dtype=torch.int32, device="cuda"),
                                  torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, keys, 0.09, window=window, want_lse=True)
    call()
    want, sums = call.out.clone(), call.lse.clone()
    assert torch.isfinite(want).all() and torch.isfinite(sums).all()
    rows = sorted({0, 1, n // 2, min(59, n - 1)})
    q[rows, 2, 5] = float("nan")
    call()
    assert torch.isnan(call.out[rows, 2]).all() and torch.isnan(call.lse[rows, 2]).all()
    for got, before in ((call.out, want), (call.lse, sums)):
        got[rows, 2] = before[rows, 2] = 0
        assert torch.equal(got, before)


@pytest.mark.parametrize("of_values", [False, True])
@pytest.mark.parametrize("size", [float("nan"), float("inf")])
@pytest.mark.parametrize("n, keys, window", [(5, 130, 0), (40, 90, 0), (40, 130, 0), (9, 200, 30), (300, 400, 100)])
def test_a_scale_that_is_no_number_reaches_only_rows_that_see_its_block(B, n, keys, window, size, of_values):
    """The last block, which the first queries do not see, and one that only those of a window see."""
    g = _gen(n + keys)
    cache = _random_cache(B, g, 40, 2, 16, 64)
    q = torch.randn((n, 4, 64), generator=g).half().cuda()
    call = B.PreparedKV8Attention(q, cache, torch.arange(40, dtype=torch.int32, device="cuda")[None], torch.tensor([keys], dtype=torch.int32, device="cuda"),
                                  torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, keys, 0.09, window=window, want_lse=True)
    call()
    want, sums = call.out.clone(), call.lse.clone()
    at = keys - n + torch.arange(n)
    for block in ((keys - 1) // 16, (keys - n) // 16 + 1):
        scales = cache.v_scale if of_values else cache.k_scale
        kept = scales.clone()
        scales[block, 1] = size
        call()
        scales.copy_(kept)
        sees = (at >= 16 * block) & ((at - window < 16 * block + 15) if window else (at >= 0))
        assert sees.any() and not sees.all()
        other = (~sees).cuda()
        assert torch.isnan(call.out[sees.cuda(), 2:]).all() and torch.isnan(call.lse[sees.cuda(), 2:]).all()
        for got, before in ((call.out, want), (call.lse, sums)):
            assert torch.equal(got[:, :2], before[:, :2]) and torch.equal(got[other], before[other])
