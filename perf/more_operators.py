"""What a decoder's layer needs for prompts and for positions without a table: what is measured of it, in plain torch and through the library.

A decoder that takes prompts of thousands of tokens has products that are bound by operations, and wants positions that no table of
embeddings ends.  Five kinds of work:

  quantize   fp16 / bf16 rows to microscaled 4-bit floating point (E2M1 numbers, one power of two for each 32 of a row) and the
             values that the codes stand for.
  linear     the product of two such operands, bias, optional GELU: prompts, batches, a few tokens; "from_x" quantizes the
             activations on the way.
  a16        few tokens as they are (fp16 / bf16) times such weights.
  rotary     queries turned by their positions: neighbouring features or halves of a head, a part of it or all, for long contexts.
  append     keys turned by their positions and values into the 8-bit cache, the step's queries turned as well, and the touched blocks
             read back.

An operand in 4 bits is codes [ceil(K / 128), rows, 64] (row r's numbers 128 c .. 128 c + 127 in q[c, r], number 2j in the low four bits of
byte j; sign, two bits of exponent, one of mantissa; zeros behind K) and scales [ceil(K / 128), rows] in words of four: byte j of word
[c, r] is 127 + the exponent of row r's numbers 128 c + 32 j and the 31 after.
"""
import math
import random

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # a few tokens of a decoding step: launch and latency
        {"name": "quantize_3x1024", "kind": "quantize", "M": 3, "K": 1024, "dtype": "bf16"},
        # the wide activations of a batch of prompts
        {"name": "quantize_12288x4096", "kind": "quantize", "M": 12288, "K": 4096, "dtype": "fp16"},
        # a few tokens through a square projection
        {"name": "linear_5x1024x1024", "kind": "linear", "M": 5, "N": 1024, "K": 1024, "from_x": False, "gelu": False, "dtype": "fp16"},
        # one short prompt, a row length that is no multiple of what kernels like
        {"name": "linear_301x4096x1056", "kind": "linear", "M": 301, "N": 4096, "K": 1056, "from_x": False, "gelu": False, "dtype": "bf16"},
        # the feed-forward layer of the larger encoder over a batch, activations quantized on the way
        {"name": "linear_12288x4096x1024_gelu", "kind": "linear", "M": 12288, "N": 4096, "K": 1024, "from_x": True, "gelu": True, "dtype": "fp16"},
        # long prompts through a wide layer: bound by operations
        {"name": "linear_7000x7424x8192", "kind": "linear", "M": 7000, "N": 7424, "K": 8192, "from_x": False, "gelu": False, "dtype": "bf16"},
        # one token, weights alone count
        {"name": "a16_1x4096x4096", "kind": "a16", "M": 1, "N": 4096, "K": 4096, "gelu": False, "dtype": "bf16"},
        # a full batch of single tokens through a wide layer
        {"name": "a16_32x16000x4096_gelu", "kind": "a16", "M": 32, "N": 16000, "K": 4096, "gelu": True, "dtype": "fp16"},
        # the queries of one decoding step, halves of a head
        {"name": "rotary_16x12x64", "kind": "rotary", "tokens": 16, "heads": 12, "D": 64, "part": 1.0, "interleaved": False, "scaling": "none",
         "context": 2048, "dtype": "fp16"},
        # prompts far into a long context, neighbouring features, frequencies scaled by parts
        {"name": "rotary_8191x32x128_parts", "kind": "rotary", "tokens": 8191, "heads": 32, "D": 128, "part": 1.0, "interleaved": True, "scaling": "parts",
         "context": 500000, "dtype": "bf16"},
        # one token for each request of a batch, with its queries
        {"name": "append_decode_48", "kind": "append", "requests": 48, "new": 1, "heads": 8, "group": 4, "D": 128, "part": 1.0, "interleaved": False,
         "block": 32, "dtype": "bf16"},
        # prompts of several thousand tokens together, odd lengths, some behind an earlier part, half of each head turned
        {"name": "append_prompt_3x4001", "kind": "append", "requests": 3, "new": 4001, "heads": 8, "group": 4, "D": 128, "part": 0.5, "interleaved": False,
         "block": 16, "dtype": "fp16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantize", "linear", "linear", "linear", "a16", "a16", "rotary", "append", "append"))
    dtype = rng.choice(("fp16", "bf16"))
    if kind == "quantize":
        K = 32 * _log_uniform(rng, 1, 400)
        return {"kind": kind, "M": _log_uniform(rng, 1, min(20000, 50_000_000 // K)), "K": K, "dtype": dtype}
    if kind == "linear":
        N, K = 8 * _log_uniform(rng, 8, 2000), 32 * _log_uniform(rng, 4, 350)
        return {"kind": kind, "M": _log_uniform(rng, 1, min(20000, int(8.4e11 / 2 / N / K))), "N": N, "K": K, "from_x": rng.random() < 0.4,
                "gelu": rng.random() < 0.3, "dtype": dtype}
    if kind == "a16":
        return {"kind": kind, "M": _log_uniform(rng, 1, 64), "N": 8 * _log_uniform(rng, 8, 2000), "K": 32 * _log_uniform(rng, 4, 350),
                "gelu": rng.random() < 0.3, "dtype": dtype}
    D, part, interleaved = rng.choice((64, 96, 128, 256)), rng.choice((1.0, 1.0, 0.5, 0.25)), rng.random() < 0.5
    if kind == "rotary":
        heads = rng.choice((1, 2, 5, 8, 12, 16, 32))
        return {"kind": kind, "tokens": _log_uniform(rng, 1, 33_000_000 // (heads * D)), "heads": heads, "D": D, "part": part, "interleaved": interleaved,
                "scaling": rng.choice(("none", "linear", "parts")), "context": _log_uniform(rng, 1000, 1_000_000), "dtype": dtype}
    heads, new = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 3, _log_uniform(rng, 20, 3000)))
    group = rng.choice((1, 2, 4, 5))
    most = max(2, 12000 * 8 * 128 * 6 // (new * heads * D * (group + 2))) if new > 3 else 200
    return {"kind": kind, "requests": _log_uniform(rng, 1, min(200, most)), "new": new, "heads": heads, "group": group, "D": D, "part": part,
            "interleaved": interleaved, "block": rng.choice((16, 32, 64, 128)), "dtype": dtype}


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

    def activations(self, M, K, dtype):
        """Rows whose ranges differ, with a few channels that are wider than the others."""
        x = self.normal((M, K)) * torch.exp(self.normal((M, 1), std=0.5))
        x[:, torch.randperm(K, generator=self.g, device="cuda")[:max(1, K // 200)]] *= 12
        return x.to(dtype)


def _spread(n, lo, hi):
    """n whole numbers over lo .. hi in no order, hi among them: the same ones for every seed, so that outputs keep their shapes."""
    values = [hi - (hi - lo) * i // n for i in range(n)]
    return random.Random(n + 1000 * hi).sample(values, n)


# ---- 4-bit operands ----------------------------------------------------------------------------------------------------
def _grid(x):
    """Magnitudes (of 4-bit numbers' indices, 0 .. 7) nearest to |x|, ties to the even one, and the exponents of blocks: x [rows, K] in fp32."""
    blocks = x.view(x.shape[0], -1, 32)
    exponent = (torch.frexp(blocks.abs().amax(-1, keepdim=True))[1] - 3).clamp(-127, 127)
    a = torch.ldexp(blocks.abs(), -exponent).clamp(max=6.0)
    index = torch.where(a < 2, torch.round(2 * a), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4))
    return index.int(), exponent


def _planes(x):
    """x [rows, n, ...] with rows and groups of four of the n in each other's place, zeros behind the last: [ceil(n / 4), rows, 4, ...]."""
    rows, n = x.shape[:2]
    full = torch.zeros((rows, (n + 3) // 4 * 4, *x.shape[2:]), dtype=x.dtype, device="cuda")
    full[:, :n] = x
    return full.view(rows, -1, 4, *x.shape[2:]).transpose(0, 1).contiguous()


def _operand(x):
    """Codes and scale words of x [rows, K]: a layer's weights, or activations that an earlier call has quantized."""
    x = x.float()
    index, exponent = _grid(x)
    codes = (index + 8 * torch.signbit(x).view(index.shape)).to(torch.uint8)
    return {"q": _planes(codes[..., 0::2] | codes[..., 1::2] << 4).flatten(2), "K": x.shape[1],
            "scale": _planes((exponent[..., 0] + 127).to(torch.uint8)).view(torch.int32)[..., 0].contiguous()}


def _prepare_quantize(case, r):
    s = {"kind": "quantize", "X": r.activations(case["M"], case["K"], DTYPES[case["dtype"]])}
    if own:
        from paper_2301_12017_amd import binding as B
        quantize = B.PreparedMX4Quantize(s["X"])
        s["calls"] = [quantize, B.PreparedMX4Dequantize(quantize.out, s["X"].dtype)]
    return s


def _weights(case, r):
    return _operand(r.normal((case["N"], case["K"]), std=0.03) * r.uniform((case["N"], 1), 0.5, 2.0))


def _prepare_linear(case, r):
    dtype = DTYPES[case["dtype"]]
    X = r.activations(case["M"], case["K"], dtype)
    s = {"kind": "linear", "W": _weights(case, r), "bias": r.normal((case["N"],), dtype, 0.1), "gelu": case["gelu"], "dtype": dtype}
    s.update({"X": X} if case["from_x"] else {"A": _operand(X)})
    if own:
        from paper_2301_12017_amd import binding as B
        act = B.ACT_GELU if case["gelu"] else B.ACT_NONE
        first = [B.PreparedMX4Quantize(X)] if case["from_x"] else []
        A = first[0].out if first else B.MX4(s["A"]["q"], s["A"]["scale"], case["K"])
        s["calls"] = first + [B.PreparedMX4Linear(A, B.MX4(s["W"]["q"], s["W"]["scale"], case["K"]), s["bias"], act, dtype)]
    return s


def _prepare_a16(case, r):
    dtype = DTYPES[case["dtype"]]
    s = {"kind": "a16", "X": r.activations(case["M"], case["K"], dtype), "W": _weights(case, r), "bias": r.normal((case["N"],), dtype, 0.1),
         "gelu": case["gelu"], "dtype": dtype}
    if own:
        from paper_2301_12017_amd import binding as B
        s["calls"] = [B.PreparedMX4LinearA16(s["X"], B.MX4(s["W"]["q"], s["W"]["scale"], case["K"]), s["bias"], B.ACT_GELU if case["gelu"] else B.ACT_NONE)]
    return s


# ---- positions ---------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians that a position turns each pair of features by, in 64 bits, and what cosines and sines are multiplied by."""
    pairs, scaling, factor, trained = int(case["D"] * case["part"]) // 2, case.get("scaling", "none"), 8.0, 8192
    f = [10000.0 ** (-i / pairs) for i in range(pairs)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":                                                        # pairs that turn often stay, those that hardly turn are slowed
        keep = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - 1) / 31)) for x in f]
        f = [x * k + x / factor * (1 - k) for x, k in zip(f, keep)]
    return torch.tensor(f, dtype=torch.float64, device="cuda"), 0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0


def _prepare_rotary(case, r):
    T, H, D, dtype = case["tokens"], case["heads"], case["D"], DTYPES[case["dtype"]]
    f, magnitude = _frequencies(case)
    starts = r.integers((T,), 0, max(1, case["context"] - T))                     # prompts of 1000 tokens from different places on, padding between
    at = torch.arange(T, device="cuda")
    positions = starts[at // 1000 * 1000] + at.int() % 1000 if T > 200 else starts
    positions = torch.where(at % 997 == 996, -1, positions).int()
    fused = r.normal((T, (H + 2) * D), dtype, 1.2)                                # the queries of a fused projection
    s = {"kind": "rotary", "x": fused[:, :H * D].view(T, H, D), "positions": positions, "f": f, "interleaved": case["interleaved"], "magnitude": magnitude}
    if own:
        from paper_2301_12017_amd import binding as B
        s["call"] = B.PreparedRotary(s["x"], positions, B.RotaryAngles(f, case["interleaved"], magnitude))
    return s


def _blocks_of(tokens, block):
    return (tokens + block - 1) // block


def _prepare_append(case, r):
    R, H, G, D, block, dtype = case["requests"], case["heads"], case["group"] * case["heads"], case["D"], case["block"], DTYPES[case["dtype"]]
    count = [case["new"]] * R if case["new"] <= 3 else _spread(R, case["new"] // 2, case["new"])
    had = [0 if i % 5 == 4 else n for i, n in enumerate(_spread(R, 0, 4 * block - 1))]
    at = r.order(R).long()
    old, new = (torch.tensor(c, dtype=torch.int32, device="cuda")[at] for c in (had, count))
    have = _blocks_of(old + new, block)
    ids = r.order(int(have.sum()) + 3)                                            # blocks in no order
    base = (torch.cumsum(have, 0) - have).long()

    def tokens_of(first, n):
        """Places in their requests of n tokens each from `first` on, and their slots."""
        total = int(n.sum())
        which = torch.repeat_interleave(torch.arange(R, device="cuda"), n.long(), output_size=total)
        pos = torch.arange(total, device="cuda") - (torch.cumsum(n, 0) - n)[which] + first[which]
        return pos.int(), (ids[base[which] + pos // block] * block + pos % block).int()

    positions, slots = tokens_of(old, new)
    _, seen = tokens_of(old // block * block, old + new - old // block * block)   # what a reader of the touched blocks reads
    f, magnitude = _frequencies(case)
    T, blocks = slots.numel(), ids.numel()
    fused = r.normal((T, (G + 2 * H) * D), dtype, 1.2)                            # queries, keys and values as a fused projection leaves them
    q, k, v = (x.view(T, -1, D) for x in fused.split([G * D, H * D, H * D], 1))
    s = {"kind": "append", "q": q, "K": k, "V": v, "slots": slots, "positions": positions, "seen": seen, "block": block, "f": f,
         "interleaved": case["interleaved"], "magnitude": magnitude,
         "k": r.integers((blocks, H, block, D), -127, 128, torch.int8), "v": r.integers((blocks, H, D, block), -127, 128, torch.int8),
         "k_scale": r.uniform((blocks, H), 0.02, 0.04), "v_scale": r.uniform((blocks, H), 0.02, 0.04)}
    if own:
        from paper_2301_12017_amd import binding as B
        cache = B.KVCache8(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["calls"] = [B.PreparedKV8AppendRotary(cache, k, v, slots, positions, B.RotaryAngles(f, case["interleaved"], magnitude), q),
                      B.PreparedKV8Read(cache, seen, dtype)]
    return s


def prepare(case, seed):
    made = {"quantize": _prepare_quantize, "linear": _prepare_linear, "a16": _prepare_a16, "rotary": _prepare_rotary, "append": _prepare_append}
    return made[case["kind"]](case, _Draws(seed))


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _values(Q):
    """The numbers [rows, K] that codes and scales stand for, in fp32."""
    q, rows = Q["q"].to(torch.int32), Q["q"].shape[1]
    codes = torch.stack([q & 15, q >> 4], -1).view(-1, rows, 4, 32)
    exponent = Q["scale"][..., None].contiguous().view(torch.uint8).int() - 127
    v = torch.tensor([*E2M1, *(-x for x in E2M1)], device="cuda")[codes]
    return torch.ldexp(v, exponent[..., None]).transpose(0, 1).reshape(rows, -1)[:, :Q["K"]]


def _plain_quantize(x):
    x = x.float()
    index, exponent = _grid(x)
    v = torch.ldexp(torch.tensor(E2M1, device="cuda")[index], exponent).view(x.shape)
    return torch.where(x < 0, -v, v)


def _plain_linear(s):
    X = s["X"].float() if s["kind"] == "a16" else _plain_quantize(s["X"]) if "X" in s else _values(s["A"])
    y = X @ _values(s["W"]).t() + s["bias"].float()
    if s["gelu"]:
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y.to(s["dtype"])


def _turned(x, s):
    """x [tokens, heads, features] turned by the tokens' positions, in fp32; tokens of a negative position as they are."""
    pairs = s["f"].numel()
    angle = s["positions"].double()[:, None] * s["f"]
    cos, sin = ((g(angle) * s["magnitude"]).float()[:, None] for g in (torch.cos, torch.sin))
    x = x.float()
    part, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
    a, b = (part[..., 0::2], part[..., 1::2]) if s["interleaved"] else (part[..., :pairs], part[..., pairs:])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.where((s["positions"] >= 0)[:, None, None], torch.cat([part, rest], -1), x)


def _plain_store(x, codes, scale, block, slots, seen):
    """New rows x [T, heads, features] in fp32 into codes [blocks, heads, block, features] (a view), then the rows of `seen`."""
    blocks, H = scale.shape
    T, at, off = slots.numel(), (slots // block).long(), (slots % block).long()
    wide = torch.zeros((blocks, H), device="cuda").scatter_reduce(0, at[:, None].expand(T, H), x.abs().amax(-1), "amax")
    first = torch.full((blocks,), block, device="cuda").scatter_reduce(0, at, off, "amin")
    was = torch.where((first == 0)[:, None], 0.0, scale)
    now = torch.maximum(was, wide / 127.0)
    now = torch.where(now < 2.0 ** -126, 0.0, now)
    now = torch.where((first < block)[:, None], now, scale)
    ratio = torch.where((first < block)[:, None], torch.where(now > 0, was / now, 0.0), 1.0)
    sat, soff = (seen // block).long(), (seen % block).long()
    codes[sat, :, soff] = (codes[sat, :, soff].float() * ratio[sat][:, :, None]).round().to(torch.int8)
    inv = torch.where(now > 0, 1.0 / now, 0.0)
    codes[at, :, off] = (x * inv[at][:, :, None]).round().clamp(-127, 127).to(torch.int8)
    scale.copy_(now)
    return codes[sat, :, soff].float() * now[sat][:, :, None]


def _plain_append(s):
    dtype = s["K"].dtype
    k = _plain_store(_turned(s["K"], s), s["k"], s["k_scale"], s["block"], s["slots"], s["seen"])
    v = _plain_store(s["V"].float(), s["v"].transpose(2, 3), s["v_scale"], s["block"], s["slots"], s["seen"])
    return {"q": _turned(s["q"], s).to(dtype), "k": k.to(dtype), "v": v.to(dtype), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    kind = state["kind"]
    if kind == "quantize":
        if own:
            quantize, dequantize = state["calls"]
            quantize()
            dequantize()
            return dequantize.out
        return _plain_quantize(state["X"]).to(state["X"].dtype)
    if kind in ("linear", "a16"):
        if own:
            for call in state["calls"]:
                call()
            return state["calls"][-1].out
        return _plain_linear(state)
    if kind == "rotary":
        if own:
            state["call"]()
            return state["call"].out
        return _turned(state["x"], state).to(state["x"].dtype)
    if own:
        append, read = state["calls"]
        append()
        read()
        return {"q": append.q, "k": read.k, "v": read.v, "k_scale": state["k_scale"], "v_scale": state["v_scale"]}
    return _plain_append(state)


def work(case):
    """Bytes of inputs and outputs, each once, and operations."""
    kind = case["kind"]
    if kind == "quantize":                                                        # rows in; codes and scales out and in again; values out
        return {"bytes": case["M"] * case["K"] * (2 + 2 * 17 / 32 + 2), "flops": 4 * case["M"] * case["K"]}
    if kind in ("linear", "a16"):
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K * 17 / 32 + M * K * (2 if kind == "a16" or case["from_x"] else 17 / 32) + 2 * N + 2 * M * N, "flops": 2 * M * N * K}
    if kind == "rotary":
        n = case["tokens"] * case["heads"] * case["D"]
        return {"bytes": 4 * n + 4 * case["tokens"] + 8 * case["D"] * case["part"] / 2, "flops": 3 * n * case["part"]}
    R, H, G, D, block = case["requests"], case["heads"], case["heads"] * case["group"], case["D"], case["block"]
    T = R * (case["new"] if case["new"] <= 3 else 0.75 * case["new"])
    seen = T + R * 0.4 * block                                                    # of new tokens and of those before them in their block
    return {"bytes": 4 * T * G * D + 2 * H * D * (2 * T + T + (seen - T) + 2 * seen) + 8 * T + 4 * seen + 8 * H * seen / block,
            "flops": 3 * T * (G + H) * D * case["part"] + 4 * H * D * seen}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"quantize": lambda s: _exact_rounded(s["X"]), "linear": _exact_linear, "a16": _exact_linear, "rotary": lambda s: _exact_turned(s["x"], s),
            "append": _exact_append}[case["kind"]](s)


def _exact_rounded(x):
    """Each number of x at the nearest of its block's sixteen, halfway cases at the one whose mantissa bit is 0."""
    x = x.double()
    out = torch.empty_like(x)
    for part, to in zip(x.split(2048), out.split(2048)):
        b = part.reshape(-1, 32)
        most = b.abs().amax(1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(torch.where(most > 0, most, 1.0))) - 2)
        a = b.abs() / unit
        found = torch.zeros_like(a)
        for i in range(7):                                                        # from each number of the grid to the next one
            middle = (E2M1[i] + E2M1[i + 1]) / 2
            found += (E2M1[i + 1] - E2M1[i]) * ((a > middle) | ((a == middle) & (i % 2 == 1)))
        to.copy_((torch.sign(b) * found * unit).view(part.shape))
    return out


def _exact_operand(Q):
    q, rows = Q["q"], Q["q"].shape[1]
    out = torch.empty((rows, Q["K"]), dtype=torch.float64, device="cuda")
    for j in range(Q["K"] // 32):
        byte = torch.bitwise_right_shift(Q["scale"][j // 4], 8 * (j % 4)) & 255
        for parity in (0, 1):
            c = q[j // 4, :, 16 * (j % 4):16 * (j % 4) + 16]
            c = c // 16 if parity else c % 16
            e, m = (c // 2 % 4).double(), (c % 2).double()
            v = torch.where(c >= 8, -1.0, 1.0) * torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e - 1))
            out[:, 32 * j + parity:32 * j + 32:2] = v * torch.exp2(byte.double() - 127)[:, None]
    return out


def _exact_linear(s):
    x = s["X"].double() if s["kind"] == "a16" else _exact_rounded(s["X"]) if "X" in s else _exact_operand(s["A"])
    y = torch.matmul(x, _exact_operand(s["W"]).t().contiguous()) + s["bias"].double()
    return y * torch.special.ndtr(y) if s["gelu"] else y


def _exact_turned(x, s):
    x, pairs = x.double(), s["f"].numel()
    out = x.clone()
    for i in range(pairs):
        at = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + pairs)
        angle = torch.remainder(s["positions"].double() * s["f"][i], 2 * math.pi)
        turn = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None]
        z = torch.complex(x[..., at[0]].contiguous(), x[..., at[1]].contiguous()) * turn
        there = (s["positions"] >= 0)[:, None]
        for place, part in zip(at, (z.real, z.imag)):
            out[..., place] = torch.where(there, part, x[..., place])
    return out


def _exact_append(s):
    block = s["block"]
    got = {"q": _exact_turned(s["q"], s)}
    place = torch.full((s["k"].shape[0] * block,), -1, dtype=torch.long, device="cuda")
    place[s["slots"].long()] = torch.arange(s["slots"].numel(), device="cuda")    # which new token a slot takes
    owner = place.view(-1, block)
    written = owner >= 0
    for name, rows, codes, scale in (("k", _exact_turned(s["K"], s), s["k"].permute(0, 2, 1, 3), s["k_scale"]),
                                     ("v", s["V"].double(), s["v"].permute(0, 3, 1, 2), s["v_scale"])):
        new = scale.double().clone()
        for b in written.any(1).nonzero()[:, 0].split(512):
            w = written[b]
            values = torch.where(w[..., None, None], rows[owner[b].clamp(min=0)], 0.0)               # [blocks, block, H, D]
            new[b] = torch.maximum(torch.where(w[:, :1], 0.0, scale[b].double()), values.abs().amax(dim=(1, 3)) / 127)
        at, off = (s["seen"] // block).long(), (s["seen"] % block).long()
        token, step = owner[at, off], new[at][..., None]
        old = torch.round(codes[at, off].double() * scale[at].double()[..., None] / step) * step
        fill = torch.round(rows[token.clamp(min=0)] / step) * step
        got[name] = torch.where((token >= 0)[:, None, None], fill, old)
        got[name + "_scale"] = new
    return {name: got[name] for name in ("q", "k", "v", "k_scale", "v_scale")}
