"""The decoder of paper_2301_12017_amd/decoder.py: every operator of token generation as it is used, against float64."""
import math

import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def _deq(W):
    """float64 [N, K] of a QWeight in canonical codes."""
    q = W.q.cpu().to(torch.int32)
    c = torch.stack([q & 15, q >> 4], -1).view(W.N, -1)
    c = torch.where(c > 7, c - 16, c) if W.mode == 0 else c
    c = c.double().view(W.N, W.scale.shape[1], -1) * W.scale.cpu().double()[:, :, None]
    return (c if W.zero is None else c + W.zero.cpu().double()[:, :, None]).view(W.N, W.K)


def _ln(x, ln, eps):
    mean, var = x.mean(1, keepdim=True), x.var(1, unbiased=False, keepdim=True)
    return (x - mean) / torch.sqrt(var + eps) * ln[0].cpu().double() + ln[1].cpu().double()


def _layer(B, layer, x, history, n, lens, table):
    """One layer in float64 on what its cache holds (keys and values are those of the cache: their 8 bits are tested by themselves)."""
    D, H, G = layer.features, layer.kv_heads, layer.heads
    b = [t.cpu().double() for t in layer.bias]
    qkv = x @ _deq(layer.qkv).t() + b[0]
    q = qkv[:, :G * D].view(-1, G, D)
    out, at = torch.zeros_like(q), 0
    for r, (a, L) in enumerate(zip(n, lens)):
        pos = torch.arange(L)
        slots = (table[r, pos // layer.cache.block] * layer.cache.block + pos % layer.cache.block).int().cuda()
        k, v = (t.cpu().double() for t in B.kv8_read(layer.cache, slots, torch.float16))
        for head in range(G):
            s = q[at:at + a, head] @ k[:, head // (G // H)].t() * D ** -0.5
            s = torch.where(pos[None] <= (L - a + torch.arange(a))[:, None], s, -math.inf)
            out[at:at + a, head] = torch.softmax(s, 1) @ v[:, head // (G // H)]
        at += a
    y = _ln(out.reshape(len(x), -1) @ _deq(layer.out).t() + b[1] + x, layer.ln1, layer.eps)
    h = y @ _deq(layer.ffn1).t() + b[2]
    h = 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    return _ln(h @ _deq(layer.ffn2).t() + b[3] + y, layer.ln2, layer.eps)


@pytest.mark.parametrize("mode,group,hidden,heads,kv_heads,block", [(0, 128, 768, 12, 4, 16), (1, 64, 512, 4, 1, 32), (0, 0, 384, 4, 4, 16)])
def test_decoder_steps(mode, group, hidden, heads, kv_heads, block):
    """Prompts, then single tokens, a request that ends and one that begins in its blocks, a row without tokens."""
    from paper_2301_12017_amd import binding as B, decoder as dec
    d = dec.random_decoder(2, hidden, heads, kv_heads, 1024, 500, requests=4, context=256, block=block, group=group, mode=mode, seed=hidden)
    g = torch.Generator().manual_seed(1)
    want_lens = [0] * 4
    for new in ([70, 1, 33, 0], [1, 1, 1, 0], [2, 1, 5, 9], [1, -1, 1, 1], [1, 40, 1, 1]):
        n = [max(a, 0) for a in new]
        want_lens = [0 if a < 0 else L + a for a, L in zip(new, want_lens)]
        ids = torch.randint(0, 500, (sum(n),), generator=g)
        got, plan = d.step(ids.cuda(), torch.tensor(new, dtype=torch.int32).cuda(), max(n))
        torch.cuda.synchronize()
        assert plan.lens.tolist() == want_lens
        table = d.books.table.cpu()
        pos = torch.cat([torch.arange(L - a, L) for a, L in zip(n, want_lens)])
        assert torch.equal(plan.positions.cpu().long(), pos)
        x = (d.tokens.cpu()[ids] + d.positions.cpu()[pos]).double()
        for layer in d.layers:
            x = _layer(B, layer, x, None, n, want_lens, table)
        # six results a layer are rounded to fp16 (2^-11 each); what enters a LayerNorm is about as large as what leaves it
        assert (got.cpu().double() - x).norm() <= 2 * 6 * 2.0 ** -11 * 2 * x.norm()
    logits = d.logits(got)
    assert logits.shape == (len(got), 500)
    assert (logits.cpu().double() - got.cpu().double() @ _deq(d.head)[:500].t()).norm() <= 2.0 ** -10 * logits.double().norm().cpu()


def test_decoder_generates_what_it_would_step_by_step():
    from paper_2301_12017_amd import decoder as dec
    prompts = [torch.arange(5) * 7, torch.arange(40) * 3, torch.arange(1)]
    a = dec.random_decoder(requests=3, context=128, seed=3)
    found = a.generate(prompts, 6)
    b = dec.random_decoder(requests=3, context=128, seed=3)
    ids, n = torch.cat(prompts).cuda(), [len(p) for p in prompts]
    for i in range(6):
        x, plan = b.step(ids, torch.tensor(n, dtype=torch.int32).cuda(), max(n))
        last = x[(plan.start[1:] - 1).long()].contiguous()
        ids = b.logits(last).argmax(1)
        assert torch.equal(ids, found[:, i])
        n = [1, 1, 1]
