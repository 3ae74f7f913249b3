"""A small decoder that writes one token at a time, from the library's operators of token generation.

Its layers are the encoder's (post-LayerNorm, GELU feed-forward) with causal attention over an 8-bit cache:

    x  = LN1(x + attn_out(attention(qkv(x))))        qkv, attn_out, ffn1, ffn2: w4a4_linear_w4a16 (4-bit weights, fp16 activations)
    x  = LN2(x + ffn2(gelu(ffn1(x))))                attention: w4a4_kv8_append, w4a4_kv8_attention

Weights may be in microscaled 4-bit floating point instead (weights="mx4"): single tokens and logits go through w4a4_mx4_linear_a16, the activations of prompts are
quantized too and go through w4a4_mx4_linear (`activations`: when, if at all).  Positions come from a table of embeddings, or queries and keys are turned by them (angles: w4a4_kv8_append_rotary).

A step takes any number of new tokens of each request (a prompt, a few, one, none, or the end of a request); w4a4_kv8_plan keeps the books of
blocks on the device.  All layers share one block table.  `python -m paper_2301_12017_amd.decoder` runs random weights.
"""
import torch

from . import binding as B


class Books:
    """Which blocks the requests of a batch own: lengths, block table and the ring of free blocks, all on the device.  A request holds up to
    `context` tokens, rounded up to whole blocks."""

    def __init__(self, requests: int, context: int, blocks: int, block=16, device="cuda"):
        z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
        width = -(-context // block)
        self.block, self.context = block, width * block
        self.table, self.ring = z(requests, width), torch.arange(blocks, dtype=torch.int32, device=device)
        self.lens, self.state = [z(requests), z(requests)], [torch.tensor([0, blocks], dtype=torch.int32, device=device), z(2)]
        self.now = 0                                       # which of the two holds the present
        self.workspace = B.KV8Workspace()                  # of the layers' attention, one after the other

    def plan(self, new_tokens: torch.Tensor, tokens: int) -> B.PreparedKV8Plan:
        """Books `new_tokens` [requests] (negative: the request has ended), `tokens` of them at most."""
        i, self.now = self.now, 1 - self.now
        call = B.PreparedKV8Plan(self.lens[i], new_tokens, self.table, self.ring, self.state[i], self.block, tokens,
                                 lens_out=self.lens[1 - i], state_out=self.state[1 - i])
        call()
        return call


# Tokens of a step up to which microscaled weights meet activations as they are, whatever they are: the weights are read again for every 16 or 32 of them.  us of the product
# with 16-bit activations | of quantizer and product: 4096 x 4096 16 tokens 5.2 | 6.8, 64 9.3 | 7.0, 128 12.8 | 9.1, 512 42 | 14; 32000 x 768 64 tokens 13 | 7, 512 82 | 15.
FEW = 64

# When more of them are quantized: in steps where a request has several new tokens ("prompts"; all rows of such a step are), so that steps of single tokens do not depend on how many
# requests there are; never ("16 bits"); always ("4 bits").  Quantizing a row moves its numbers by up to a quarter of them, or of its block's power of two.  Rows of logits are never quantized.
ACTIVATIONS = ("prompts", "16 bits", "4 bits")


def quantized(W: torch.Tensor, weights="int4", mode=None, group=None):
    """W [N, K] (fp16) in the 4-bit form asked for: integer codes ("int4", symmetric ones in groups of 128 where nothing else is said) or microscaled floating
    point ("mx4", which has neither modes nor groups)."""
    if weights not in ("int4", "mx4"):
        raise ValueError(f"weights {weights!r}: int4 or mx4")
    if weights == "int4":
        return B.quantize_weight(W, B.SYM if mode is None else mode, 128 if group is None else group)
    if mode is not None or group is not None:
        raise ValueError(f"mode {mode}, group {group}: microscaled weights have blocks of 32 and no mode")
    return B.mx4_quantize(W)


def linear(x: torch.Tensor, W, bias=None, act=B.ACT_NONE, exact=True) -> torch.Tensor:
    """x [tokens, K] (fp16) times what `quantized` made.  exact: x as it is; else more than FEW rows are quantized where the weights are microscaled."""
    if isinstance(W, B.QWeight):
        return B.linear_w4a16(x, W, bias, act)
    if exact or len(x) <= FEW:
        return B.mx4_linear_a16(x, W, bias, act)
    return B.mx4_linear(B.mx4_quantize(x), W, bias, act, x.dtype)


class DecoderLayer:
    """One layer: 4-bit weights (see `quantized`), a cache of `blocks` blocks.  heads: of queries; kv_heads: of keys and values (grouped heads).  angles: what
    queries and keys are turned by (RotaryAngles), None where positions are in the embeddings.  activations: one of ACTIVATIONS, of microscaled weights."""

    def __init__(self, Wqkv, bqkv, Wo, bo, W1, b1, W2, b2, g1, be1, g2, be2, heads: int, kv_heads: int, blocks: int, block=16, group=None, mode=None, eps=1e-12,
                 weights="int4", angles=None, activations="prompts"):
        if activations not in ACTIVATIONS:
            raise ValueError(f"activations {activations!r}: one of {ACTIVATIONS}")
        hidden, self.activations = Wo.shape[0], activations
        self.heads, self.kv_heads, self.features, self.eps = heads, kv_heads, Wo.shape[1] // heads, eps
        assert Wqkv.shape == ((heads + 2 * kv_heads) * self.features, hidden)
        self.qkv, self.out, self.ffn1, self.ffn2 = (quantized(W, weights, mode, group) for W in (Wqkv, Wo, W1, W2))
        self.bias = (bqkv, bo, b1, b2)
        self.ln1, self.ln2, self.angles = (g1, be1), (g2, be2), angles
        self.cache = B.KVCache8.new(blocks, kv_heads, self.features, block, device=Wo.device)

    def __call__(self, x: torch.Tensor, books: Books, plan: B.PreparedKV8Plan, queries: int) -> torch.Tensor:
        T, D = x.shape[0], self.features
        exact = self.activations == "16 bits" or self.activations == "prompts" and queries <= 1
        q, k, v = (t.view(T, -1, D) for t in linear(x, self.qkv, self.bias[0], exact=exact).split([self.heads * D, self.kv_heads * D, self.kv_heads * D], 1))
        if self.angles is None:
            B.kv8_append(self.cache, k, v, plan.slots)
        else:
            q = B.kv8_append_rotary(self.cache, k, v, plan.slots, plan.positions, self.angles, q)
        a = B.kv8_attention(q, self.cache, books.table, plan.lens, plan.start, queries, books.context, D ** -0.5, workspace=books.workspace)
        x = self._norm(linear(a.view(T, -1), self.out, self.bias[1], exact=exact), x, self.ln1)
        h = linear(x, self.ffn1, self.bias[2], B.ACT_GELU, exact)
        return self._norm(linear(h, self.ffn2, self.bias[3], exact=exact), x, self.ln2)

    def _norm(self, x, residual, ln):
        return B.layernorm_quantize(x, residual, ln[0], ln[1], self.eps)[1]


class Decoder:
    """Token and position embeddings (positions None: the layers turn queries and keys), layers, and the logits of the tokens' successors from the
    quantized token embeddings."""

    def __init__(self, layers, tokens: torch.Tensor, positions, books: Books, group=None, weights="int4"):
        if positions is None and not all(layer.angles for layer in layers):
            raise ValueError("no position embeddings, and layers without angles")
        if positions is not None and len(positions) < books.context:       # (the plan hands out every position of a block, and they are looked up unseen)
            raise ValueError(f"{len(positions)} position embeddings for requests of up to {books.context} tokens")
        self.layers, self.tokens, self.positions, self.books = layers, tokens, positions, books
        pad = -len(tokens) % 8                             # (the linear's channels come in eights)
        self.head = quantized(torch.nn.functional.pad(tokens, (0, 0, 0, pad)).contiguous(), weights, None, group)

    def step(self, ids: torch.Tensor, new_tokens: torch.Tensor, queries: int):
        """ids [tokens]: the new tokens of all requests, one after the other, new_tokens [requests] of them each and `queries` at most.  Returns the
        hidden states [tokens, hidden] and the plan; tokens of requests that found no blocks hold nothing that means anything."""
        plan = self.books.plan(new_tokens, ids.numel())
        x = self.tokens[ids]
        if self.positions is not None:
            x = x + self.positions[plan.positions.clamp(min=0).long()]
        for layer in self.layers if len(x) else ():        # (a step in which requests only end has no tokens)
            x = layer(x, self.books, plan, queries)
        return x, plan

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        return linear(x, self.head)[:, :len(self.tokens)]

    def generate(self, prompts, new: int) -> torch.Tensor:
        """The `new` likeliest next tokens [requests, new], one at a time, behind prompts (a list of 1-D tensors of ids, one or more each).  Requests
        go on from what they hold, and end with the call: their blocks are free again.  Raises where a request found no blocks, or
        no room in its context."""
        dev, n = self.tokens.device, [len(p) for p in prompts]
        if len(n) != self.books.lens[0].numel() or not all(n) or new < 1:
            raise ValueError(f"prompts of {n} tokens, {new} new ones: one prompt for each of {self.books.lens[0].numel()} requests, at least a token each")
        if max(n) + new - 1 > self.books.context:
            raise ValueError(f"{max(n)} tokens and {new - 1} behind them do not fit a context of {self.books.context}")
        ids, new_tokens = torch.cat([p.to(dev) for p in prompts]).long(), torch.tensor(n, dtype=torch.int32, device=dev)
        one, queries, found = torch.ones_like(new_tokens), max(n), []
        served = torch.ones((), dtype=torch.bool, device=dev)              # (looked at once, behind the last step: nothing waits for it)
        for _ in range(new):
            x, plan = self.step(ids, new_tokens, queries)
            last = (plan.start[1:] - 1).long()
            served &= (plan.positions[last] >= 0).all()
            ids = self.logits(x[last].contiguous()).argmax(1)
            found.append(ids)
            new_tokens, queries = one, 1
        self.step(ids[:0], -one, 1)
        if not served:
            raise RuntimeError("a request was not served: too few free blocks, or its context was full")
        return torch.stack(found, 1)


def random_decoder(layers=2, hidden=768, heads=12, kv_heads=4, ffn=2048, vocabulary=1000, requests=4, context=512, block=16, group=None, mode=None, seed=0,
                   weights="int4", rotary=False, activations="prompts") -> Decoder:
    """Random weights of the given sizes, and blocks for `requests` requests of `context` tokens.  rotary: no position embeddings, queries and keys turn."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, std=0.02: (torch.randn(shape, generator=g, device="cuda") * std).half()
    D, blocks = hidden // heads, requests * -(-context // block)
    books = Books(requests, context, blocks, block)
    angles = B.RotaryAngles(B.rotary_frequencies(D // 2)[0]) if rotary else None
    one = lambda: (1 + normal(hidden, std=0.05).float()).half()
    made = [DecoderLayer(normal((heads + 2 * kv_heads) * D, hidden, std=0.05), normal((heads + 2 * kv_heads) * D), normal(hidden, heads * D), normal(hidden),
                         normal(ffn, hidden), normal(ffn), normal(hidden, ffn), normal(hidden), one(), normal(hidden), one(), normal(hidden),
                         heads, kv_heads, blocks, block, group, mode, weights=weights, angles=angles,
                         activations=activations) for _ in range(layers)]
    return Decoder(made, normal(vocabulary, hidden, std=1.0), None if rotary else normal(books.context, hidden, std=0.3), books, group, weights)


if __name__ == "__main__":
    import time
    draw = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 32000, (100 + 37 * i,), generator=draw) for i in range(16)]
    for kind in ({}, {"weights": "mx4", "rotary": True}):
        decoder = random_decoder(layers=12, ffn=4096, vocabulary=32000, requests=16, context=2048, **kind)
        took = []
        for new in (1, 64):
            decoder.generate(prompts, new)
            torch.cuda.synchronize()
            began = time.perf_counter()
            found = decoder.generate(prompts, new)
            torch.cuda.synchronize()
            took.append(time.perf_counter() - began)
        print(f"{kind.get('weights', 'int4')}{', rotary' if kind else ''}: 12 layers of 768, 16 requests of 100 to 655 tokens: prompts and their first tokens in "
              f"{1e3 * took[0]:.1f} ms, {found.numel()} tokens in {took[1]:.3f} s ({found.numel() / took[1]:.0f} a second), prompts included")
