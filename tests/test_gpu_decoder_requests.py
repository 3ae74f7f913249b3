"""Decoder.generate: one call after the other."""
import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]

PROMPTS = [torch.arange(5) * 7, torch.arange(40) * 3, torch.arange(1)]


def _decoder(**kw):
    from paper_2301_12017_amd import decoder as dec
    return dec.random_decoder(hidden=256, heads=4, kv_heads=2, ffn=512, requests=3, seed=3, **{"context": 128, **kw})


def test_generate_again_begins_anew():
    d = _decoder()
    first, again = d.generate(PROMPTS, 6), d.generate(PROMPTS, 6)
    assert torch.equal(first, again) and torch.equal(first, _decoder().generate(PROMPTS, 6))
    assert d.books.lens[d.books.now].tolist() == [0, 0, 0] and int(d.books.state[d.books.now][1]) == d.books.ring.numel()
    more = torch.arange(3).mul(11)
    assert torch.equal(d.generate([more] * 3, 4), _decoder().generate([more] * 3, 4))
