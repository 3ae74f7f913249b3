"""Operators of token generation: what is measured of them, in plain torch and through the library.

A decoder that writes one token at a time reads its weights and its cache and computes little.  Four kinds of work:

  linear     fp16 / bf16 activations of a few tokens times 4-bit weights (per channel or per K-group, symmetric or
             unsigned codes in the canonical packing), bias, optional GELU.
  plan       the block bookkeeping of one step: new blocks from the ring of free ones, the block table, one cache slot and
             one position per new token, blocks of ended requests back into the ring.
  append     keys and values of new tokens into the 8-bit cache, one scale per block and head (a block whose range grows is
             re-scaled), and the touched blocks read back.
  attention  queries over that cache: single tokens, a few per request, or a whole prompt; grouped heads, causal, with or
             without a window.

The cache holds K codes as [blocks, heads, block, features], V codes as [blocks, heads, features, block] and a scale for
each block and head; block tables name the blocks of a request in order.
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # one token through a projection of the smaller encoder's size: launch and latency
        {"name": "linear_1x768x768", "kind": "linear", "M": 1, "N": 768, "K": 768, "group": 0, "asym": False, "dtype": "fp16", "gelu": False},
        # a small ragged batch through a square projection, groups of 128
        {"name": "linear_5x4096x4096_g128", "kind": "linear", "M": 5, "N": 4096, "K": 4096, "group": 128, "asym": False, "dtype": "bf16", "gelu": False},
        # a full batch through a wide feed-forward layer, unsigned codes
        {"name": "linear_32x16384x4096_u128", "kind": "linear", "M": 32, "N": 16384, "K": 4096, "group": 128, "asym": True, "dtype": "fp16", "gelu": True},
        # one decoding step of a batch: one token for each request, some of them done
        {"name": "plan_decode_64", "kind": "plan", "requests": 64, "new": 1, "context": 4096, "block": 32},
        # many requests at once, prompts among them, the ring nearly empty
        {"name": "plan_mixed_2999", "kind": "plan", "requests": 2999, "new": 300, "context": 8192, "block": 16},
        # one token for each request of a batch
        {"name": "append_decode_48", "kind": "append", "requests": 48, "new": 1, "heads": 8, "D": 128, "block": 32, "dtype": "bf16"},
        # prompts of several thousand tokens together, odd lengths, some behind an earlier part
        {"name": "append_prompt_5x3001", "kind": "append", "requests": 5, "new": 3001, "heads": 8, "D": 128, "block": 16, "dtype": "fp16"},
        # one short conversation, every head with its own keys
        {"name": "attention_1x777", "kind": "attention", "requests": 1, "queries": 1, "context": 777, "heads": 12, "kv_heads": 12, "D": 64, "block": 16, "window": 0, "dtype": "fp16"},
        # a batch of ragged conversations, grouped heads: the ordinary decoding step (the last request is a padding row)
        {"name": "attention_32x5000", "kind": "attention", "requests": 32, "queries": 1, "context": 5000, "heads": 32, "kv_heads": 8, "D": 128, "block": 32, "window": 0, "dtype": "bf16"},
        # one very long document: the keys have to be shared out
        {"name": "attention_1x150001", "kind": "attention", "requests": 1, "queries": 1, "context": 150001, "heads": 32, "kv_heads": 8, "D": 128, "block": 64, "window": 0, "dtype": "fp16"},
        # a few drafted tokens per request, a sliding window, an odd number of query heads per key head
        {"name": "attention_7x4_window", "kind": "attention", "requests": 7, "queries": 4, "context": 2500, "heads": 10, "kv_heads": 2, "D": 96, "block": 16, "window": 1000, "dtype": "bf16"},
        # the last part of a prompt behind an earlier part
        {"name": "attention_prompt_2x1500", "kind": "attention", "requests": 2, "queries": 1500, "context": 4100, "heads": 32, "kv_heads": 8, "D": 128, "block": 32, "window": 0, "dtype": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "linear", "plan", "append", "attention", "attention", "attention"))
    dtype = rng.choice(("fp16", "bf16"))
    if kind == "linear":
        asym, group = rng.random() < 0.4, rng.choice((0, 32, 64, 96, 128, 128, 256))
        k = _log_uniform(rng, 256, 11000)
        K = max(1, k // (group or 32)) * (group or 32)
        return {"kind": kind, "M": _log_uniform(rng, 1, 64), "N": 8 * _log_uniform(rng, 16, 2000), "K": K, "group": group, "asym": asym,
                "dtype": dtype, "gelu": rng.random() < 0.3}
    if kind == "plan":
        return {"kind": kind, "requests": _log_uniform(rng, 1, 3000), "new": rng.choice((1, 1, 4, 60, 300)), "context": _log_uniform(rng, 500, 8192),
                "block": rng.choice((16, 32, 64, 128))}
    heads, D, block = rng.choice((1, 2, 4, 8, 12)), rng.choice((64, 96, 128, 256)), rng.choice((16, 32, 64, 128))
    if kind == "append":
        new = rng.choice((1, 1, 3, _log_uniform(rng, 20, 3000)))
        return {"kind": kind, "requests": _log_uniform(rng, 1, max(2, 12000 // new if new > 3 else 200)), "new": new, "heads": heads, "D": D,
                "block": block, "dtype": dtype}
    group, queries = rng.choice((1, 1, 2, 4, 5, 7, 8, 16)), rng.choice((1, 1, 1, 2, 5, _log_uniform(rng, 16, 1500)))
    while heads * group * D > 8192:
        heads = max(1, heads // 2)
        group = max(1, group // 2) if heads == 1 else group
    requests = _log_uniform(rng, 1, 40) if queries < 16 else rng.choice((1, 2))
    rows = requests * heads * group * queries
    most = min(120_000, 140_000_000 // (requests * heads * D), 250_000_000 // rows, 28_000_000_000 // (rows * D))
    context = queries + _log_uniform(rng, 30, max(60, most))
    return {"kind": kind, "requests": requests, "queries": queries, "context": context, "heads": heads * group, "kv_heads": heads, "D": D,
            "block": block, "window": rng.choice((0, 0, 0, 17, 900)), "dtype": dtype}


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * std).to(dtype)

    def uniform(self, shape, lo, hi):
        return torch.rand(shape, generator=self.g, device="cuda") * (hi - lo) + lo

    def integers(self, shape, lo, hi, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda").int()

    def shuffled(self, *columns):
        """The rows of these columns in another order."""
        at = self.order(len(columns[0])).long()
        return [torch.tensor(c, dtype=torch.int32, device="cuda")[at] for c in columns]


def _spread(n, lo, hi):
    """n whole numbers over lo .. hi in no order, hi among them: the same ones for every seed, so that outputs keep their shapes."""
    values = [hi - (hi - lo) * i // n for i in range(n)]
    return random.Random(n + 1000 * hi).sample(values, n)


def _lengths(case):
    """Queries and keys of each request of an attention case, in the order before it is shuffled."""
    Q, C, pad = case["queries"], case["context"], case["requests"] >= 4           # (a row that pads the batch: one query, nothing to see)
    n = _spread(case["requests"] - pad, 1, Q)
    lens = [Q + more - (Q - a) // 2 for a, more in zip(n, _spread(case["requests"] - pad, 0, C - Q))]
    lens[0] = C
    return n + [1] * pad, lens + [0] * pad


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _prepare_linear(case, r):
    M, N, K, group, dtype = case["M"], case["N"], case["K"], case["group"], DTYPES[case["dtype"]]
    ng = K // group if group else 1
    codes = (r.normal((N, K // 2, 2), std=2.4) + (7.5 if case["asym"] else 0.0)).round()
    codes = codes.clamp(0, 15) if case["asym"] else codes.clamp(-7, 7)
    codes = codes.to(torch.int32) & 15
    s = {"kind": "linear", "X": r.normal((M, K), dtype), "q": (codes[..., 0] | codes[..., 1] << 4).to(torch.uint8),
         "scale": r.uniform((N, ng), 0.5, 1.5) * 0.008, "zero": None, "bias": r.normal((N,), dtype, 0.1), "group": group,
         "gelu": case["gelu"]}
    s["X"][:, torch.randperm(K, generator=r.g, device="cuda")[:4]] *= 8          # a few channels with a wide range
    if case["asym"]:
        s["zero"] = s["scale"] * -r.uniform((N, ng), 6.5, 8.5)
    if own:
        from paper_2301_12017_amd import binding as B
        W = B.QWeight(s["q"], s["scale"], s["zero"], None, None, N, K, group, B.ASYM if case["asym"] else B.SYM)
        s["call"] = B.PreparedLinearW4A16(s["X"], W, s["bias"], B.ACT_GELU if case["gelu"] else B.ACT_NONE)
    return s


def _blocks_of(tokens, block):
    return (tokens + block - 1) // block


def _table(r, lens, block, width, spare):
    """Block tables with blocks in no order, what lies behind a request's last block left as it may be; the blocks over."""
    have = _blocks_of(lens, block)
    n = int(have.sum())
    ids = r.order(n + spare)
    first = (torch.cumsum(have, 0) - have)[:, None]
    col = torch.arange(width, device="cuda")[None]
    table = torch.where(col < have[:, None], ids[(first + col).clamp(max=n + spare - 1).long()], 0x7FFFFFF0)
    return table.int().contiguous(), ids[n:].contiguous(), n + spare


def _prepare_plan(case, r):
    R, block = case["requests"], case["block"]
    few = [1] * R if case["new"] == 1 else [n if i % 10 < 3 else 1 for i, n in enumerate(_spread(R, 0, case["new"]))]
    few = [-1 if i % 33 == 32 else n for i, n in enumerate(few)]                 # some requests have ended
    lens = _spread(R, 0, case["context"])
    wanted = sum(_blocks_of(a + n, block) - _blocks_of(a, block) for a, n in zip(lens, few) if n > 0)
    lens, new = r.shuffled(lens, few)
    width = _blocks_of(case["context"] + case["new"], block)
    table, spare, blocks = _table(r, lens, block, width, int(wanted * 0.97) + 8 if case["new"] == 300 else wanted + 40)
    ring = torch.empty(blocks, dtype=torch.int32, device="cuda")
    head = blocks * 2 // 3
    at = (head + torch.arange(blocks, device="cuda")) % blocks                   # the free ones from `head` on, used entries behind them
    ring[at] = torch.cat([spare, torch.full((blocks - spare.numel(),), -1, dtype=torch.int32, device="cuda")])
    s = {"kind": "plan", "lens": lens, "new": new, "table": table, "ring": ring, "block": block,
         "state": torch.tensor([head, spare.numel()], dtype=torch.int32, device="cuda"), "tokens": int(new.clamp(min=0).sum()) + 5}
    if own:
        from paper_2301_12017_amd import binding as B
        s["call"] = B.PreparedKV8Plan(lens, new, table, ring, s["state"], block, s["tokens"])
    return s


def _prepare_append(case, r):
    R, H, D, block, dtype = case["requests"], case["heads"], case["D"], case["block"], DTYPES[case["dtype"]]
    new = [case["new"]] * R if case["new"] <= 3 else _spread(R, case["new"] // 2, case["new"])
    old, new = r.shuffled([0 if i % 5 == 4 else n for i, n in enumerate(_spread(R, 0, 4 * block - 1))], new)
    lens = old + new
    width = int(_blocks_of(lens, block).max())
    table, _, blocks = _table(r, lens, block, width, 3)
    T = int(new.sum())
    which = torch.repeat_interleave(torch.arange(R, device="cuda"), new.long(), output_size=T)
    pos = torch.arange(T, device="cuda") - (torch.cumsum(new, 0) - new)[which] + old[which]
    slots = (table[which, pos // block] * block + pos % block).int()
    # what a reader of the touched blocks reads: from the first token of the first touched block on
    first = old // block * block
    n = lens - first
    S = int(n.sum())
    which = torch.repeat_interleave(torch.arange(R, device="cuda"), n.long(), output_size=S)
    pos = torch.arange(S, device="cuda") - (torch.cumsum(n, 0) - n)[which] + first[which]
    seen = (table[which, pos // block] * block + pos % block).int()
    fused = r.normal((T, 3 * H * D), dtype)                                      # keys and values as a fused projection leaves them
    k, v = fused[:, H * D:2 * H * D].view(T, H, D), fused[:, 2 * H * D:].view(T, H, D)
    s = {"kind": "append", "K": k, "V": v, "slots": slots, "seen": seen, "block": block, "dtype": dtype,
         "k": r.integers((blocks, H, block, D), -127, 128, torch.int8), "v": r.integers((blocks, H, D, block), -127, 128, torch.int8),
         "k_scale": r.uniform((blocks, H), 0.015, 0.03), "v_scale": r.uniform((blocks, H), 0.015, 0.03)}
    if own:
        from paper_2301_12017_amd import binding as B
        cache = B.KVCache8(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["calls"] = [B.PreparedKV8Append(cache, k, v, slots), B.PreparedKV8Read(cache, seen, dtype)]
    return s


def _codes(r, shape, channels, dim):
    """int8 codes of about normal values, some of the `channels` shifted, as keys have them."""
    side = [1] * len(shape)
    side[1], side[dim] = shape[1], channels
    c = r.normal(shape, std=30.0) + r.normal((shape[1], channels), std=10.0).view(side)
    return c.round_().clamp_(-127, 127).to(torch.int8)


def _prepare_attention(case, r):
    R, H, G, D, block, dtype = case["requests"], case["kv_heads"], case["heads"], case["D"], case["block"], DTYPES[case["dtype"]]
    n, lens = r.shuffled(*_lengths(case))
    width = _blocks_of(case["context"], block)
    table, _, blocks = _table(r, lens, block, width, 2)
    T = int(n.sum())
    fused = r.normal((T, (G + 2 * H) * D), dtype, 1.2)                           # the queries of a fused projection
    s = {"kind": "attention", "q": fused[:, :G * D].view(T, G, D), "start": torch.cat([n.new_zeros(1), torch.cumsum(n, 0)]).int(), "lens": lens.int(),
         "table": table, "k": _codes(r, (blocks, H, block, D), D, 3), "v": _codes(r, (blocks, H, D, block), D, 2),
         "k_scale": r.uniform((blocks, H), 0.02, 0.04), "v_scale": r.uniform((blocks, H), 0.01, 0.05), "block": block,
         "queries": case["queries"], "context": case["context"], "window": case["window"], "scale": D ** -0.5}
    if own:
        from paper_2301_12017_amd import binding as B
        cache = B.KVCache8(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["call"] = B.PreparedKV8Attention(s["q"], cache, table, s["lens"], s["start"], case["queries"], case["context"], s["scale"],
                                           window=case["window"], want_lse=True)
    return s


def prepare(case, seed):
    return {"linear": _prepare_linear, "plan": _prepare_plan, "append": _prepare_append, "attention": _prepare_attention}[case["kind"]](case, _Draws(seed))


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _plain_linear(s):
    N, K = s["q"].shape[0], 2 * s["q"].shape[1]
    q = s["q"].to(torch.int32)
    codes = torch.stack([q & 15, q >> 4], -1).view(N, s["scale"].shape[1], -1)
    if s["zero"] is None:
        w = (codes - 16 * (codes >> 3)).float() * s["scale"][:, :, None]
    else:
        w = codes.float() * s["scale"][:, :, None] + s["zero"][:, :, None]
    y = s["X"].float() @ w.view(N, K).t() + s["bias"].float()
    if s["gelu"]:
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["X"].dtype)


def _plain_plan(s):
    lens, new, table, ring, block = s["lens"], s["new"], s["table"], s["ring"], s["block"]
    width, cap = table.shape[1], ring.numel()
    head, free = s["state"][0], s["state"][1]
    ended, add = new < 0, new.clamp(min=0)
    after = lens + add
    bad = (lens < 0) | (lens > width * block)
    have, full = (lens + block - 1) // block, (after + block - 1) // block
    fits = ~bad & ~ended & (after <= width * block)
    need = torch.where(fits, full - have, 0)
    upto = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (upto <= free))
    col = torch.arange(width, device="cuda")[None]
    take = (head + (upto - need)[:, None] + col - have[:, None]) % cap
    table = torch.where(served[:, None] & (col >= have[:, None]) & (col < full[:, None]), ring[take], table)
    give = ended & ~bad
    back = torch.where(give, have, 0)
    to = (head + free + (torch.cumsum(back, 0) - back)[:, None] + col) % cap
    to = torch.where(give[:, None] & (col < have[:, None]), to, cap)
    ring = torch.cat([ring, ring[:1]]).scatter(0, to.reshape(-1), table.reshape(-1))[:cap]
    taken = torch.where(served, need, 0).sum()
    state = torch.stack([(head + taken) % cap, free - taken + back.sum()]).int()
    total = torch.cumsum(add, 0)
    t = torch.arange(s["tokens"], device="cuda")
    r = torch.searchsorted(total, t, right=True).clamp(max=lens.numel() - 1)
    pos = lens[r] + t - (total - add)[r]
    there = (t < total[-1]) & served[r]
    slot = table[r, (pos // block).clamp(0, width - 1)] * block + pos % block
    return {"table": table, "ring": ring, "state": state, "lens": torch.where(give, 0, torch.where(served, after, lens)).int(),
            "start": torch.cat([total.new_zeros(1), total]).int(), "slots": torch.where(there, slot, -1).int(),
            "positions": torch.where(there, pos, -1).int()}


def _plain_store(x, codes, scale, block, slots, seen):
    """New rows x [T, heads, features] into codes [blocks, heads, block, features] (a view), then the rows of `seen`."""
    blocks, H = scale.shape
    T, at, off = slots.numel(), (slots // block).long(), (slots % block).long()
    x = x.float()
    wide = torch.zeros((blocks, H), device="cuda").scatter_reduce(0, at[:, None].expand(T, H), x.abs().amax(-1), "amax")
    first = torch.full((blocks,), block, device="cuda").scatter_reduce(0, at, off, "amin")
    was = torch.where((first == 0)[:, None], 0.0, scale)
    now = torch.maximum(was, wide / 127.0)
    now = torch.where(now < 2.0 ** -126, 0.0, now)
    now = torch.where((first < block)[:, None], now, scale)
    ratio = torch.where(now > 0, was / now, 0.0)
    ratio = torch.where((first < block)[:, None], ratio, 1.0)
    sat, soff = (seen // block).long(), (seen % block).long()
    codes[sat, :, soff] = (codes[sat, :, soff].float() * ratio[sat][:, :, None]).round().to(torch.int8)
    inv = torch.where(now > 0, 1.0 / now, 0.0)
    codes[at, :, off] = (x * inv[at][:, :, None]).round().clamp(-127, 127).to(torch.int8)
    scale.copy_(now)
    return codes[sat, :, soff].float() * now[sat][:, :, None]


def _plain_append(s):
    k = _plain_store(s["K"], s["k"], s["k_scale"], s["block"], s["slots"], s["seen"])
    v = _plain_store(s["V"], s["v"].transpose(2, 3), s["v_scale"], s["block"], s["slots"], s["seen"])
    return {"k": k.to(s["dtype"]), "v": v.to(s["dtype"]), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attention(s):
    block, lens, R = s["block"], s["lens"], s["lens"].numel()
    T, G, D = s["q"].shape
    H = s["k"].shape[1]
    n = s["start"][1:] - s["start"][:-1]
    ids = s["table"][:, :(s["context"] + block - 1) // block].clamp(0, s["k"].shape[0] - 1).long()
    L = ids.shape[1] * block
    there = torch.arange(L, device="cuda") < lens[:, None]                       # [R, L]
    k = s["k"][ids].float() * s["k_scale"][ids][..., None, None]                 # [R, blocks, H, block, D]
    k = torch.where(there[:, None, :, None], k.permute(0, 2, 1, 3, 4).reshape(R, H, L, D), 0.0)
    v = s["v"][ids].float() * s["v_scale"][ids][..., None, None]                 # [R, blocks, H, D, block]
    v = torch.where(there[:, None, :, None], v.permute(0, 2, 1, 4, 3).reshape(R, H, L, D), 0.0)
    j = torch.arange(s["queries"], device="cuda")
    row = (s["start"][:-1, None] + j).clamp(max=T - 1).long()                    # [R, queries]
    q = s["q"][row].float().view(R, -1, H, G // H, D).permute(0, 2, 1, 3, 4).reshape(R, H, -1, D)
    x = (q @ k.transpose(2, 3)).view(R, H, -1, G // H, L) * s["scale"]
    at = (lens[:, None] - n[:, None] + j)[:, None, :, None, None]                # position of each query
    t = torch.arange(L, device="cuda")
    sees = t <= at
    if s["window"]:
        sees = sees & (t > at - s["window"])
    x = torch.where(sees, x, -math.inf)
    most = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(most == -math.inf, 0.0, most))
    total = p.sum(-1, keepdim=True)
    o = (p.view(R, H, -1, L) @ v).view(R, H, -1, G // H, D) / torch.where(total == 0, 1.0, total)
    lse = (most + torch.log(total))[..., 0]                                      # [R, H, queries, G / H]
    r = torch.searchsorted(s["start"][1:].contiguous(), torch.arange(T, dtype=torch.int32, device="cuda"), right=True)
    i = torch.arange(T, device="cuda") - s["start"][r]
    return {"out": o[r, :, i].reshape(T, G, D).to(s["q"].dtype), "lse": lse[r, :, i].reshape(T, G)}


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    kind = state["kind"]
    if kind == "linear":
        if own:
            state["call"]()
            return state["call"].out
        return _plain_linear(state)
    if kind == "plan":
        if own:
            call = state["call"]
            call()
            return {"table": state["table"], "ring": state["ring"], "state": call.state, "lens": call.lens, "start": call.start,
                    "slots": call.slots, "positions": call.positions}
        return _plain_plan(state)
    if kind == "append":
        if own:
            append, read = state["calls"]
            append()
            read()
            return {"k": read.k, "v": read.v, "k_scale": state["k_scale"], "v_scale": state["v_scale"]}
        return _plain_append(state)
    if own:
        state["call"]()
        return {"out": state["call"].out, "lse": state["call"].lse}
    return _plain_attention(state)


def work(case):
    """Bytes of inputs and outputs, each once, and operations."""
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        ng = K // case["group"] if case["group"] else 1
        return {"bytes": N * K / 2 + N * ng * (8 if case["asym"] else 4) + 2 * N + 2 * M * (K + N), "flops": 2 * M * N * K}
    if case["kind"] == "plan":
        R, new = case["requests"], 1 if case["new"] == 1 else 0.7 + 0.15 * case["new"]
        width = _blocks_of(case["context"] + case["new"], case["block"])
        # lengths in and out, starts; a slot and a position per token; new table entries; the blocks of ended requests
        return {"bytes": R * (16 + 8 * new + 8 * new / case["block"] + 0.03 * 8 * width / 2), "flops": R * new * 4}
    if case["kind"] == "append":
        R, H, D, block = case["requests"], case["heads"], case["D"], case["block"]
        T = R * (case["new"] if case["new"] <= 3 else 0.75 * case["new"])
        seen = T + R * 0.4 * block                                                # of new tokens and of those before them in their block
        return {"bytes": 2 * H * D * (2 * T + T + (seen - T) + 2 * seen) + 4 * T + 4 * seen + 8 * H * seen / block, "flops": 4 * H * D * seen}
    H, G, D, W = case["kv_heads"], case["heads"], case["D"], case["window"]
    keys = pairs = queries = 0
    for n, length in zip(*_lengths(case)):
        seen = min(length, W + n - 1) if W else length                           # keys that any of the queries sees
        keys, queries = keys + seen, queries + n
        pairs += sum(min(p + 1, W) if W else p + 1 for p in range(length - n, length)) if length else 0
    return {"bytes": keys * H * (2 * D + 8 / case["block"]) + 4 * keys / case["block"] + queries * G * (4 * D + 4), "flops": 4 * D * G * pairs}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "plan": lambda s: None, "append": _exact_append, "attention": _exact_attention}[case["kind"]](s)


def _exact_linear(s):
    X, q = s["X"].double(), s["q"]
    N, half = q.shape
    group = s["group"] or 2 * half
    out = torch.zeros((X.shape[0], N), dtype=torch.float64, device="cuda")
    for g in range(2 * half // group):
        part = q[:, g * group // 2:(g + 1) * group // 2].long()
        for parity in (0, 1):
            c = (part >> (4 * parity)) % 16
            if s["zero"] is None:
                c = torch.where(c > 7, c - 16, c)
            x = X[:, g * group + parity:(g + 1) * group:2].contiguous()
            out += (x @ c.double().t().contiguous()) * s["scale"][:, g].double()
            if s["zero"] is not None:
                out += x.sum(1, keepdim=True) * s["zero"][:, g].double()
    out += s["bias"].double()
    return out * torch.special.ndtr(out) if s["gelu"] else out


def _exact_append(s):
    block, got = s["block"], {}
    place = torch.full((s["k"].shape[0] * block,), -1, dtype=torch.long, device="cuda")
    place[s["slots"].long()] = torch.arange(s["slots"].numel(), device="cuda")   # which new token a slot takes
    owner = place.view(-1, block)
    written = owner >= 0
    for name, rows, codes, scale in (("k", s["K"], s["k"].permute(0, 2, 1, 3), s["k_scale"]), ("v", s["V"], s["v"].permute(0, 3, 1, 2), s["v_scale"])):
        fresh = torch.zeros(scale.shape, dtype=torch.float64, device="cuda")
        new = scale.double().clone()
        for b in written.any(1).nonzero()[:, 0].split(512):
            w = written[b]
            values = torch.where(w[..., None, None], rows[owner[b].clamp(min=0)].double(), 0.0)      # [blocks, block, H, D]
            before = torch.where(w[:, :1], fresh[b], scale[b].double())
            new[b] = torch.maximum(before, values.abs().amax(dim=(1, 3)) / 127)
        got[name + "_scale"] = new
        at, off = (s["seen"] // block).long(), (s["seen"] % block).long()
        token = owner[at, off]
        step = new[at][..., None]
        old = torch.round(codes[at, off].double() * scale[at].double()[..., None] / step) * step
        fill = torch.round(rows[token.clamp(min=0)].double() / step) * step
        got[name] = torch.where((token >= 0)[:, None, None], fill, old)
    return got


def _exact_attention(s):
    T, G, D = s["q"].shape
    H, block = s["k"].shape[1], s["block"]
    out = torch.zeros((T, G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((T, G), -math.inf, dtype=torch.float64, device="cuda")
    start, lens = s["start"].tolist(), s["lens"].tolist()
    for r, length in enumerate(lens):
        a, b = start[r], start[r + 1]
        ids = s["table"][r, :(length + block - 1) // block].long()
        if not length or a == b:
            continue
        for h in range(H):
            k = (s["k"][ids, h].double() * s["k_scale"][ids, h].double()[:, None, None]).reshape(-1, D)[:length]
            v = (s["v"][ids, h].double() * s["v_scale"][ids, h].double()[:, None, None]).transpose(1, 2).reshape(-1, D)[:length]
            q = s["q"][a:b, h * (G // H):(h + 1) * (G // H)].double()
            x = torch.matmul(q.reshape(-1, D), k.t().contiguous()).view(b - a, G // H, length) * s["scale"]
            age = (torch.arange(length - (b - a), length, device="cuda")[:, None] - torch.arange(length, device="cuda"))[:, None]
            x[(age < 0).expand_as(x)] = -math.inf
            if s["window"]:
                x[(age >= s["window"]).expand_as(x)] = -math.inf
            z = torch.logsumexp(x, -1)
            lse[a:b, h * (G // H):(h + 1) * (G // H)] = z
            w = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[..., None])
            out[a:b, h * (G // H):(h + 1) * (G // H)] = torch.matmul(w.view(-1, length), v).view(b - a, G // H, D)
    return {"out": out, "lse": lse}
