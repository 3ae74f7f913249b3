"""Which activations of a decoder with microscaled weights are quantized, and how far from float64 that leaves its products."""
import math

import pytest
import torch

from tests.gpu_util import has_gpu
from tests.test_gpu_decoder_mx4 import _deq, _layer

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def _check_steps(d, steps, requests):
    """Each step's rows against the layers in float64, within the roundings of activations as they are: six results a layer and the turned queries in fp16 (2^-11 each); what
    enters a LayerNorm is about as large as what leaves it.  Then the logits, which have the fp32 sums' roundings and one more."""
    from paper_2301_12017_amd import binding as B
    g, lens = torch.Generator().manual_seed(1), [0] * requests
    for n in steps:
        lens = [L + a for a, L in zip(n, lens)]
        ids = torch.randint(0, 500, (sum(n),), generator=g)
        got, plan = d.step(ids.cuda(), torch.tensor(n, dtype=torch.int32).cuda(), max(n))
        assert plan.lens.tolist() == lens
        pos = torch.cat([torch.arange(L - a, L) for a, L in zip(n, lens)])
        x = d.tokens.cpu()[ids].double()
        for layer in d.layers:
            x = _layer(B, layer, x, pos, n, lens, d.books.table.cpu())
        assert (got.cpu().double() - x).norm() <= 2 * 7 * 2.0 ** -11 * len(d.layers) * x.norm()
        logits = d.logits(got)
        assert logits.shape == (len(got), 500)
        assert (logits.cpu().double() - got.cpu().double() @ _deq(B, d.head)[:500].t()).norm() <= 2.0 ** -10 * logits.double().norm().cpu()


def test_single_tokens_of_many_requests_are_not_quantized():
    from paper_2301_12017_amd import decoder as dec
    d = dec.random_decoder(2, 256, 4, 2, 512, 500, requests=70, context=32, seed=9, weights="mx4", rotary=True)
    _check_steps(d, [[1] * 70, [1] * 70, [1] * 66 + [0] * 4], 70)


def test_prompts_are_not_quantized_where_that_is_asked_for():
    from paper_2301_12017_amd import decoder as dec
    d = dec.random_decoder(1, 768, 12, 4, 2048, 500, requests=3, context=256, seed=5, weights="mx4", rotary=True, activations="16 bits")
    _check_steps(d, [[100, 7, 50], [1, 65, 3]], 3)


def test_what_is_quantized():
    """Steps of 70 rows by the three choices: bit for bit those of the other choice that they stand for."""
    from paper_2301_12017_amd import decoder as dec
    found = {}
    for activations in dec.ACTIVATIONS:
        d = dec.random_decoder(1, 256, 4, 2, 512, 500, requests=70, context=64, seed=9, weights="mx4", rotary=True, activations=activations)
        ids = torch.arange(70).cuda()
        single, _ = d.step(ids, torch.ones(70, dtype=torch.int32).cuda(), 1)
        few = torch.zeros(70, dtype=torch.int32)
        few[:2] = torch.tensor([40, 24])
        small, _ = d.step(ids[:64], few.cuda(), 40)
        few[:2] = torch.tensor([20, 50])
        d.step(ids[:0], torch.full((70,), -1, dtype=torch.int32).cuda(), 1)
        prompt, _ = d.step(ids, few.cuda(), 50)
        found[activations] = single, small, prompt
    p, exact, quantized = (found[a] for a in ("prompts", "16 bits", "4 bits"))
    assert torch.equal(p[0], exact[0]) and not torch.equal(p[0], quantized[0])
    assert torch.equal(p[1], exact[1])                             # (up to FEW rows as they are; the cache behind "4 bits" holds other keys)
    assert torch.equal(p[2], quantized[2]) and not torch.equal(p[2], exact[2])


@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("M,N,K", [(65, 264, 768), (157, 776, 544), (600, 264, 2080)])
def test_how_far_quantized_activations_are_from_float64(M, N, K, gelu):
    """A number of a block whose largest one lies in [4, 8) units is off by half a step of E2M1: a quarter of a unit up to 2 units, half of one up to 4, one up to 6, and what it
    passes 6 by, at most a quarter of it: a quarter of itself or of the unit, whichever is more.  The bound of a product sums those; K additions of fp32, GELU's slope
    (1.13) and its own error (9e-5 and 1e-8), the rounding to fp16 (2^-11, subnormal steps of 2^-24)."""
    from paper_2301_12017_amd import binding as B, decoder as dec
    g = torch.Generator().manual_seed(M + K)
    x = (torch.randn((M, K), generator=g) * torch.exp(torch.randn((M, 1), generator=g))).half()
    W, b = dec.quantized((torch.randn((N, K), generator=g) * 0.05).half().cuda(), "mx4"), torch.randn((N,), generator=g).mul(0.1).half()
    got = dec.linear(x.cuda(), W, b.cuda(), B.ACT_GELU if gelu else B.ACT_NONE, exact=False).cpu().double()
    a, w = x.double(), _deq(B, W)
    unit = torch.exp2(torch.floor(torch.log2(a.abs().view(M, -1, 32).amax(-1))) - 2).repeat_interleave(32, 1)
    moved = torch.maximum(a.abs(), unit) / 4
    y = a @ w.t() + b.double()
    err = moved @ w.abs().t() + (K + 1) * 2.0 ** -23 * ((a.abs() + moved) @ w.abs().t() + b.double().abs())
    if gelu:
        y, err = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5))), 1.13 * err
        err = err + 9e-5 * (y.abs() + err) + 1e-8
    off = (got - y).abs()
    assert (off <= err + 2.0 ** -11 * (y.abs() + err) + 2.0 ** -25).all()
    assert off.norm() <= 0.25 * (a.abs() + unit).norm() * torch.linalg.matrix_norm(w, 2) * (1.13 if gelu else 1.0) + 2.0 ** -10 * y.norm()
    exact = dec.linear(x.cuda(), W, b.cuda(), B.ACT_GELU if gelu else B.ACT_NONE).cpu().double()
    assert (exact - y).norm() <= 2.0 ** -10 * y.norm() and (exact - y).norm() < 0.05 * off.norm()
