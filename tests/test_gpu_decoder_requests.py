"""Decoder.generate: requests that are not served, empty prompts, one call after the other."""
import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]

PROMPTS = [torch.arange(5) * 7, torch.arange(40) * 3, torch.arange(1)]


def _decoder(**kw):
    from paper_2301_12017_amd import decoder as dec
    return dec.random_decoder(hidden=256, heads=4, kv_heads=2, ffn=512, requests=3, seed=3, **{"context": 128, **kw})


def _fewer_blocks(d, blocks):
    """The ring of free blocks cut to its first `blocks`."""
    d.books.state[d.books.now][1] = blocks
    return d


def test_generate_again_begins_anew():
    d = _decoder()
    first, again = d.generate(PROMPTS, 6), d.generate(PROMPTS, 6)
    assert torch.equal(first, again) and torch.equal(first, _decoder().generate(PROMPTS, 6))
    assert d.books.lens[d.books.now].tolist() == [0, 0, 0] and int(d.books.state[d.books.now][1]) == d.books.ring.numel()
    more = torch.arange(3).mul(11)
    assert torch.equal(d.generate([more] * 3, 4), _decoder().generate([more] * 3, 4))


def test_generate_raises_where_blocks_run_out():
    for blocks, new in ((4, 2), (5, 10), (5, 14)):                 # the prompts take 1 + 3 + 1 blocks of 16; the second needs one more for its 49th token
        d = _fewer_blocks(_decoder(), blocks)
        with pytest.raises(RuntimeError):
            d.generate(PROMPTS, new)
    assert torch.equal(_fewer_blocks(_decoder(), 5).generate(PROMPTS, 9), _decoder().generate(PROMPTS, 9))


def test_generate_raises_where_the_context_is_full():
    d = _decoder(context=48)
    assert d.generate(PROMPTS, 9).shape == (3, 9)                  # 40 tokens and eight behind them
    with pytest.raises(ValueError):
        d.generate(PROMPTS, 10)
    d.step(torch.arange(4, device="cuda"), torch.tensor([0, 4, 0], dtype=torch.int32, device="cuda"), 4)
    with pytest.raises(RuntimeError):                              # (with what the request held before)
        d.generate(PROMPTS, 9)


def test_generate_refuses_prompts_that_are_none():
    d = _decoder()
    for prompts, new in (([PROMPTS[0], torch.arange(0), PROMPTS[2]], 3), ([torch.arange(0)] + PROMPTS[:2], 3), (PROMPTS[:2], 3), (PROMPTS, 0)):
        with pytest.raises(ValueError):
            d.generate(prompts, new)
    assert d.books.lens[d.books.now].tolist() == [0, 0, 0]


def test_requests_fill_their_last_block_whatever_the_context():
    d = _decoder(context=40)                                       # three blocks of 16: 48 tokens
    found = d.generate(PROMPTS, 9)
    assert torch.equal(found, _decoder(context=48).generate(PROMPTS, 9))
