"""The decoder of paper_2301_12017_amd/decoder.py with microscaled weights and rotary positions: the operators as they are used together."""
import math

import pytest
import torch

from tests.gpu_util import has_gpu
from tests.test_gpu_decoder import _ln

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def _deq(B, W):
    return B.mx4_dequantize(W).cpu().double()                     # (bf16 holds such numbers exactly)


def _turned(x, pos, angles):
    """x [T, heads, features] in float64, halves turned."""
    n = angles.pairs
    turn = torch.tensor([[(t % 2 ** 64 * p % 2 ** 64) / 2.0 ** 64 for t in angles.turns.cpu().tolist()] for p in pos.tolist()], dtype=torch.float64) * 2 * math.pi
    c, s = torch.cos(turn)[:, None], torch.sin(turn)[:, None]
    a, b = x[..., :n], x[..., n:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _layer(B, layer, x, pos, n, lens, table):
    """One layer in float64 on what its cache holds, the keys turned already."""
    D, H, G = layer.features, layer.kv_heads, layer.heads
    b = [t.cpu().double() for t in layer.bias]
    qkv = x @ _deq(B, layer.qkv).t() + b[0]
    q = _turned(qkv[:, :G * D].view(-1, G, D), pos, layer.angles)
    k_new = _turned(qkv[:, G * D:(G + H) * D].view(-1, H, D), pos, layer.angles)
    out, at = torch.zeros_like(q), 0
    for r, (a, L) in enumerate(zip(n, lens)):
        p = torch.arange(L)
        slots = (table[r, p // layer.cache.block] * layer.cache.block + p % layer.cache.block).int().cuda()
        k, v = (t.cpu().double() for t in B.kv8_read(layer.cache, slots, torch.float16))
        # the cache's keys are the turned ones: off by half a step of 1 / 127 of a block's largest number, re-scaled up to fifteen times, and fp16 before
        assert (k[L - a:] - k_new[at:at + a]).norm() <= 0.02 * k_new[at:at + a].norm() + 1e-9
        for head in range(G):
            s = q[at:at + a, head] @ k[:, head // (G // H)].t() * D ** -0.5
            s = torch.where(p[None] <= (L - a + torch.arange(a))[:, None], s, -math.inf)
            out[at:at + a, head] = torch.softmax(s, 1) @ v[:, head // (G // H)]
        at += a
    y = _ln(out.reshape(len(x), -1) @ _deq(B, layer.out).t() + b[1] + x, layer.ln1, layer.eps)
    h = y @ _deq(B, layer.ffn1).t() + b[2]
    h = 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    return _ln(h @ _deq(B, layer.ffn2).t() + b[3] + y, layer.ln2, layer.eps)


@pytest.mark.parametrize("hidden,heads,kv_heads,block", [(768, 12, 4, 16), (512, 4, 1, 32), (384, 4, 4, 16)])
def test_decoder_steps(hidden, heads, kv_heads, block):
    """Steps of up to 64 tokens, whose activations are not quantized: prompts, single tokens, a request that ends and one that begins in its blocks."""
    from paper_2301_12017_amd import binding as B, decoder as dec
    d = dec.random_decoder(2, hidden, heads, kv_heads, 1024, 500, requests=4, context=256, block=block, seed=hidden, weights="mx4", rotary=True)
    g = torch.Generator().manual_seed(1)
    want_lens = [0] * 4
    for new in ([30, 1, 33, 0], [1, 1, 1, 0], [2, 1, 5, 9], [1, -1, 1, 1], [1, 40, 1, 1]):
        n = [max(a, 0) for a in new]
        want_lens = [0 if a < 0 else L + a for a, L in zip(new, want_lens)]
        ids = torch.randint(0, 500, (sum(n),), generator=g)
        got, plan = d.step(ids.cuda(), torch.tensor(new, dtype=torch.int32).cuda(), max(n))
        torch.cuda.synchronize()
        assert plan.lens.tolist() == want_lens
        table = d.books.table.cpu()
        pos = torch.cat([torch.arange(L - a, L) for a, L in zip(n, want_lens)])
        x = d.tokens.cpu()[ids].double()
        for layer in d.layers:
            x = _layer(B, layer, x, pos, n, want_lens, table)
        # six results a layer and the turned queries are rounded to fp16 (2^-11 each); what enters a LayerNorm is about as large as what leaves it
        assert (got.cpu().double() - x).norm() <= 2 * 7 * 2.0 ** -11 * 2 * x.norm()
    logits = d.logits(got)
    assert logits.shape == (len(got), 500)
    assert (logits.cpu().double() - got.cpu().double() @ _deq(B, d.head)[:500].t()).norm() <= 2.0 ** -10 * logits.double().norm().cpu()


def test_a_prompt_goes_through_the_quantized_products():
    """More than 64 tokens: the layer is its operators one after the other, bit for bit."""
    from paper_2301_12017_amd import binding as B, decoder as dec
    d = dec.random_decoder(1, 768, 12, 4, 2048, 500, requests=3, context=256, seed=5, weights="mx4", rotary=True)
    new, T = torch.tensor([100, 7, 50], dtype=torch.int32).cuda(), 157
    ids = torch.randint(0, 500, (T,), generator=torch.Generator().manual_seed(2)).cuda()
    got, plan = d.step(ids, new, 100)
    layer, D = d.layers[0], 64
    x, cache = d.tokens[ids], B.KVCache8.new(layer.cache.blocks, 4, D, 16)
    mul = lambda y, W, bias, act=B.ACT_NONE: B.mx4_linear(B.mx4_quantize(y), W, bias, act, torch.float16)
    q, k, v = (t.view(T, -1, D) for t in mul(x, layer.qkv, layer.bias[0]).split([768, 256, 256], 1))
    q = B.kv8_append_rotary(cache, k, v, plan.slots, plan.positions, layer.angles, q)
    assert torch.equal(cache.k, layer.cache.k) and torch.equal(cache.v, layer.cache.v) and torch.equal(cache.k_scale, layer.cache.k_scale)
    a = B.kv8_attention(q, cache, d.books.table, plan.lens, plan.start, 100, d.books.context, D ** -0.5)
    x = layer._norm(mul(a.view(T, -1), layer.out, layer.bias[1]), x, layer.ln1)
    x = layer._norm(mul(mul(x, layer.ffn1, layer.bias[2], B.ACT_GELU), layer.ffn2, layer.bias[3]), x, layer.ln2)
    assert torch.equal(got, x)


def test_decoder_generates_what_it_would_step_by_step():
    from paper_2301_12017_amd import decoder as dec
    prompts = [torch.arange(5) * 7, torch.arange(100) * 3, torch.arange(1)]
    make = lambda: dec.random_decoder(requests=3, context=128, seed=3, weights="mx4", rotary=True)
    a, b = make(), make()
    found = a.generate(prompts, 6)
    ids, n = torch.cat(prompts).cuda(), [len(p) for p in prompts]
    for i in range(6):
        x, plan = b.step(ids, torch.tensor(n, dtype=torch.int32).cuda(), max(n))
        ids = b.logits(x[(plan.start[1:] - 1).long()].contiguous()).argmax(1)
        assert torch.equal(ids, found[:, i])
        n = [1, 1, 1]


def test_a_step_that_finds_no_blocks_leaves_the_cache_alone():
    """Tokens that are not served have position -1 and no slot: nothing of them is stored, and the other requests' results are as without them."""
    from paper_2301_12017_amd import decoder as dec
    one, two = (dec.random_decoder(1, 256, 4, 2, 512, 100, requests=2, context=64, seed=7, weights="mx4", rotary=True) for _ in range(2))
    for d in (one, two):
        d.books.state[0][1] = 3                                   # three free blocks of sixteen tokens
    ids = torch.arange(60).cuda()
    got, plan = one.step(ids, torch.tensor([20, 40], dtype=torch.int32).cuda(), 40)
    assert plan.positions.tolist() == list(range(20)) + [-1] * 40
    alone, _ = two.step(ids[:20], torch.tensor([20, 0], dtype=torch.int32).cuda(), 20)
    assert torch.equal(one.layers[0].cache.k, two.layers[0].cache.k) and torch.equal(one.layers[0].cache.v, two.layers[0].cache.v)
    # (the attention takes rows in other tiles: the roundings of a layer, as above, on both sides)
    assert (got[:20].double() - alone.double()).norm() <= 2 * 2 * 7 * 2.0 ** -11 * alone.double().norm()
