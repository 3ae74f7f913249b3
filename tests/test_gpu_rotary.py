"""Rotary positions on the GPU against plain implementations in 64 bits on the CPU: queries, and keys on their way into the 8-bit cache.

Angles of the reference come from whole-number arithmetic on the fractions of a turn, so far positions are exact.  A turned number is off by 2^-22 of its
pair's length at most (angle 2^-25 turns of rounding in its fp32 form, below 2^-23 in all with the series' own error; products and sum 3 half steps of
2^-24), times the magnitude, and by half a step of its type, h = finfo.eps / 2."""
import math
from fractions import Fraction

import pytest
import torch

from tests.gpu_util import has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    from paper_2301_12017_amd import binding
    binding.lib()
    return binding


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _turns(angles):
    return [t % 2 ** 64 for t in angles.turns.cpu().tolist()]


def _turned(x, positions, angles, inverse=False):
    """x [T, H, D] in 64 bits, turned, and the length of each number's pair."""
    out, size, n = x.clone(), x.abs(), angles.pairs
    turn = torch.tensor([[(t * max(p, 0) % 2 ** 64) / 2.0 ** 64 for t in _turns(angles)] for p in positions.tolist()], dtype=torch.float64) * 2 * math.pi
    c, s = angles.magnitude * torch.cos(turn)[:, None], angles.magnitude * torch.sin(turn)[:, None] * (-1 if inverse else 1)
    at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if angles.interleaved else (slice(0, n), slice(n, 2 * n))
    a, b, on = x[..., at[0]], x[..., at[1]], (positions >= 0)[:, None, None]
    out[..., at[0]], out[..., at[1]] = torch.where(on, a * c - b * s, a), torch.where(on, b * c + a * s, b)
    size[..., at[0]] = size[..., at[1]] = angles.magnitude * torch.hypot(a, b)
    return out, size


def _check(got, x, positions, angles, inverse=False):
    want, size = _turned(x.double(), positions, angles, inverse)
    h = torch.finfo(got.dtype).eps / 2
    off = (got.cpu().double() - want).abs()
    assert (off <= 2.0 ** -22 * size * (1 + h) + h * want.abs() + (2.0 ** -25 if got.dtype == torch.float16 else 0)).all(), float((off / size.clamp(min=1e-30)).max())
    same = positions < 0
    assert torch.equal(got.cpu()[same], x[same]) and torch.equal(got.cpu()[..., 2 * angles.pairs:], x[..., 2 * angles.pairs:])


POSITIONS = [0, 1, 2, -1, 7, 4095, 100000, 999983, 2 ** 24 + 1, 2 ** 30 - 7, 2 ** 31 - 1, -5, 2 ** 31 - 2, 12345678]


def _angles(B, pairs, interleaved, magnitude=1.0, base=10000.0):
    return B.RotaryAngles(B.rotary_frequencies(pairs, base)[0], interleaved, magnitude)


# ---- queries -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,pairs", [(1, 1, 8, 4), (1, 1, 64, 32), (3, 12, 64, 32), (14, 5, 96, 48), (40, 32, 128, 64), (7, 2, 256, 128), (29, 3, 80, 40), (9, 33, 128, 32),
                                         (5, 7, 96, 24), (6, 4, 128, 1), (11, 3, 64, 10), (4, 2, 72, 36), (3, 1, 256, 127), (700, 2, 64, 8), (2000, 1, 8, 1)])
def test_rotary(B, T, H, D, pairs, interleaved, dtype):
    g, t = _gen(T + D), TYPES[dtype]
    x = torch.randn((T, H, D), generator=g).to(t)
    positions = torch.tensor([POSITIONS[i % len(POSITIONS)] if i < 28 else (i * 37) % 70000 for i in range(T)], dtype=torch.int32)
    angles = _angles(B, pairs, interleaved)
    _check(B.rotary(x.cuda(), positions.cuda(), angles), x, positions, angles)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs", [64, 20])
def test_rotary_in_place_of_a_fused_projection(B, interleaved, pairs):
    """A slice of wider rows, in place, a magnitude; the rest of the rows, NaN of one kind, stays as it was."""
    T, H, D = 37, 6, 128
    wide = torch.full((T, (H + 4) * D), float("nan"), dtype=torch.bfloat16)
    x = torch.randn((T, H, D), generator=_gen(1)).bfloat16()
    wide[:, D:(H + 1) * D] = x.view(T, -1)
    positions = torch.arange(T, dtype=torch.int32) * 1009 - 1
    angles = _angles(B, pairs, interleaved, 1.25)
    dev = wide.cuda()
    view = dev[:, D:(H + 1) * D].view(T, H, D)
    before = dev.clone()
    out = B.rotary(view, positions.cuda(), angles, out=view)
    assert out.data_ptr() == view.data_ptr()
    _check(view, x, positions, angles)
    rest = torch.ones(dev.shape[1], dtype=torch.bool)
    rest[D:(H + 1) * D] = False
    assert torch.equal(dev[:, rest].view(torch.int16), before[:, rest].view(torch.int16))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pairs", [32, 9])
def test_rotary_takes_numbers_that_are_not_finite_in_their_pairs(B, interleaved, pairs):
    T, H, D = 6, 3, 64
    x = torch.randn((T, H, D), generator=_gen(2)).half()
    positions, angles = torch.arange(3, 3 + T, dtype=torch.int32), _angles(B, pairs, interleaved)
    clean = B.rotary(x.cuda(), positions.cuda(), angles).cpu()
    x[2, 1, 3], x[4, 0, 63] = float("nan"), float("inf")
    got = B.rotary(x.cuda(), positions.cuda(), angles).cpu()
    partner = 2 if interleaved else 3 + pairs
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[2, 1, 3] = bad[2, 1, partner] = True
    bad[4, 0, 63] = True
    if 2 * pairs == D:
        bad[4, 0, 62 if interleaved else 31] = True
    else:
        assert got[4, 0, 63] == float("inf")
    assert torch.equal(got[~bad], clean[~bad]) and not torch.isfinite(got[bad]).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,pairs", [(64, 32), (96, 20), (128, 64)])
def test_gradient_is_the_inverse(B, D, pairs, interleaved, dtype):
    """The formula's gradient (checked as the forward is), and differences: the sum of g y changes by the sum of dx times it.  The result is linear in x: the two sides
    differ by the roundings of y, y' and the gradient alone."""
    g, t, T, H = _gen(3), TYPES[dtype], 19, 4
    positions, angles = torch.arange(T, dtype=torch.int32) * 271 - 1, _angles(B, pairs, interleaved, 1.1)
    x, dx, gy = (torch.randn((T, H, D), generator=g).to(t) for _ in range(3))
    moved = (x.double() + dx.double()).to(t)
    step = moved.double() - x.double()
    back = B.rotary(gy.cuda(), positions.cuda(), angles, inverse=True)
    _check(back, gy, positions, angles, inverse=True)
    y0, y1 = (B.rotary(v.cuda(), positions.cuda(), angles).cpu().double() for v in (x, moved))
    h = torch.finfo(t).eps / 2 + 2.0 ** -21                       # of each number's own size, or its pair's length
    left, right = (gy.double() * (y1 - y0)).sum(), (back.cpu().double() * step).sum()
    lengths = [_turned(v.double(), positions, angles)[1] for v in (x, moved, gy)]
    room = h * ((gy.double().abs() * (lengths[0] + lengths[1])).sum() + (step.abs() * lengths[2]).sum())
    assert abs(left - right) <= room
    if dtype == "fp16":                                           # there and back
        plain = _angles(B, pairs, interleaved)
        again = B.rotary(B.rotary(x.cuda(), positions.cuda(), plain), positions.cuda(), plain, inverse=True).cpu().double()
        assert ((again - x.double()).abs() <= 2 * (h + h) * lengths[0] / 1.1).all()


def test_frequencies(B):
    """Units of 2^-64 of a turn, the nearest; the rules of scaling at their ends."""
    f, m = B.rotary_frequencies(32, 500000.0)
    assert m == 1.0 and f[0] == 1 and abs(f[31].item() - 500000.0 ** (-31 / 32)) < 1e-20
    pi = Fraction("3.14159265358979323846264338327950288419716939937510")
    a = B.RotaryAngles(torch.cat([f, torch.tensor([-0.25, 7.5, 0.0], dtype=torch.float64)]))
    for t, x in zip(_turns(a), f.tolist() + [-0.25, 7.5, 0.0]):
        off = (t - Fraction(x) / (2 * pi) * 2 ** 64) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 30)
    slow, m = B.rotary_frequencies(32, 10000.0, 8.0)
    assert m == 1.0 and torch.equal(slow * 8, B.rotary_frequencies(32)[0])
    parts, m = B.rotary_frequencies(64, 10000.0, 8.0, trained=8192)
    plain = B.rotary_frequencies(64)[0]
    turns = 8192 * plain / (2 * math.pi)
    assert abs(m - (0.1 * math.log(8) + 1)) < 1e-12
    assert torch.equal(parts[turns > 32], plain[turns > 32]) and torch.allclose(parts[turns < 1], plain[turns < 1] / 8, rtol=1e-15)
    middle = (turns > 1) & (turns < 32)
    assert ((parts < plain) & (parts > plain / 8))[middle].all()
    for bad in ({"pairs": 0}, {"pairs": 4, "base": 0.0}, {"pairs": 4, "factor": 0.5}, {"pairs": 4, "trained": -1}, {"pairs": 4, "slow": 2.0, "fast": 1.0}):
        with pytest.raises(ValueError):
            B.rotary_frequencies(**bad)
    for f, m in (([], 1.0), ([[1.0]], 1.0), ([float("nan")], 1.0), ([1.0], 0.0), ([1.0], float("inf"))):
        with pytest.raises(ValueError):
            B.RotaryAngles(f, magnitude=m)


# ---- keys on their way into the cache --------------------------------------------------------------------------------------------
def _cache(B, g, blocks, H, D, block):
    C = B.KVCache8.new(blocks, H, D, block)
    C.k.copy_(torch.randint(-127, 128, C.k.shape, generator=g))
    C.v.copy_(torch.randint(-127, 128, C.v.shape, generator=g))
    C.k_scale.copy_(torch.rand(C.k_scale.shape, generator=g) * 0.01 + 0.01)
    C.v_scale.copy_(torch.rand(C.v_scale.shape, generator=g) * 0.01 + 0.01)
    return C


def _clone(B, C):
    return B.KVCache8(C.k.clone(), C.v.clone(), C.k_scale.clone(), C.v_scale.clone())


def _same(a, b):
    return all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("k", "v", "k_scale", "v_scale"))


def _runs(g, block, runs):
    """Slots of runs (block number, first place, tokens, shuffled or not), and of tokens that are not stored."""
    slots = []
    for b, first, n, mixed in runs:
        at = torch.arange(first, first + n)
        slots += (b * block + (at[torch.randperm(n, generator=g)] if mixed else at)).tolist() if b >= 0 else [-1] * n
    return torch.tensor(slots, dtype=torch.int32)


def _stored(x, slots, codes, scale, block):
    """Codes [blocks, H, block, D] and scales after x [T, H, D] in 64 bits, and the exact quotients of the new ones."""
    codes, scale, exact = codes.double(), scale.double(), {}
    for b in sorted({s // block for s in slots.tolist() if s >= 0}):
        which = [i for i, s in enumerate(slots.tolist()) if s >= 0 and s // block == b]
        places = [slots[i].item() % block for i in which]
        was = torch.zeros_like(scale[b]) if 0 in places else scale[b].clone()
        now = torch.maximum(was, x[which].abs().amax((0, 2)) / 127)
        if 0 not in places:                                       # (what a block held that begins anew means nothing, and is left)
            codes[b] = torch.round(codes[b] * (was / now)[:, None, None])
        scale[b] = now
        for i, p in zip(which, places):
            exact[b, p] = x[i] / now[:, None]
            codes[b, :, p] = torch.round(exact[b, p])
    return codes, scale, exact


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,pairs,H,block", [(64, 32, 3, 16), (96, 48, 2, 32), (96, 20, 1, 16), (128, 64, 5, 64), (128, 32, 2, 128), (256, 128, 2, 32), (128, 13, 1, 32), (64, 8, 4, 128)])
def test_append_rotary(B, D, pairs, H, block, interleaved, dtype):
    g, t, G = _gen(D + pairs), TYPES[dtype], 2 * H + 1
    runs = [(3, 0, 1, False), (-1, 0, 2, False), (5, 2, 9, False), (0, 0, block, False), (7, block - 3, 3, True), (-1, 0, 1, False), (2, 0, min(block, 40), True), (4, 5, 1, False)]
    slots = _runs(g, block, runs)
    T = slots.numel()
    positions = torch.randint(0, 200000, (T,), generator=g).int()
    positions[1], positions[T - 1], positions[4] = -1, 2 ** 31 - 1, 0
    fused = torch.randn((T, (G + 2 * H) * D), generator=g).to(t)
    q, k, v = (x.view(T, -1, D) for x in fused.cuda().split([G * D, H * D, H * D], 1))
    C = _cache(B, g, 9, H, D, block)
    before, plain = _clone(B, C), _clone(B, C)
    angles = _angles(B, pairs, interleaved, 1.2)
    got_q = B.kv8_append_rotary(C, k, v, slots.cuda(), positions.cuda(), angles, q)
    _check(got_q, q.cpu(), positions, angles)
    B.kv8_append(plain, k, v, slots.cuda())
    assert torch.equal(C.v, plain.v) and torch.equal(C.v_scale, plain.v_scale)              # values as they always were
    x, size = _turned(k.cpu().double(), positions, angles)
    codes, scale, exact = _stored(x, slots, before.k.cpu(), before.k_scale.cpu(), block)
    got, got_scale = C.k.cpu().double(), C.k_scale.cpu().double()
    assert ((got_scale - scale).abs() <= 2.0 ** -21 * scale).all()                          # 2^-22 of the largest pair's length (up to sqrt 2 of a number), a division
    off = (got - codes).abs()
    assert off.max() <= 1
    untouched = torch.ones(9, dtype=torch.bool)
    untouched[sorted({s // block for s in slots.tolist() if s >= 0})] = False
    assert not off[untouched].any()
    for (b, p), value in exact.items():                           # a code is another one only where the quotient lies at a border: 127 * (2^-21 + 2^-22 and two roundings)
        there = off[b, :, p] > 0
        assert ((value - value.floor() - 0.5).abs()[there] <= 127 * 2.0 ** -20).all()
    old = off.clone()
    for b, p in exact:
        old[b, :, p] = 0
    ratio = (before.k_scale.cpu().double() / scale)[:, :, None, None] * before.k.cpu().double()
    assert ((ratio - ratio.floor() - 0.5).abs()[old > 0] <= 127 * 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rotary_that_turns_nothing_is_append(B, interleaved, dtype):
    """Position 0 and negative ones: the bits of w4a4_kv8_append, infinities and NaN among the numbers."""
    g, H, D, block = _gen(5), 3, 96, 32
    slots = _runs(g, block, [(1, 0, 20, False), (0, 4, 3, False), (3, 0, 32, True), (2, 31, 1, False)])
    T = slots.numel()
    k, v = (torch.randn((T, H, D), generator=g).to(TYPES[dtype]) for _ in range(2))
    k[3, 0, 5], k[30, 1, 70], k[31, 2, 0], v[8, 0, 1] = float("nan"), float("inf"), -float("inf"), float("nan")
    C = _cache(B, g, 4, H, D, block)
    plain = _clone(B, C)
    B.kv8_append(plain, k.cuda(), v.cuda(), slots.cuda())
    assert B.kv8_append_rotary(C, k.cuda(), v.cuda(), slots.cuda(), torch.full((T,), -1, dtype=torch.int32).cuda(), _angles(B, 40, interleaved)) is None
    assert _same(C, plain)
    k = torch.nan_to_num(k, 1.0, 2.0, -2.0)                       # (an infinity times the sine of 0 is NaN)
    C = _cache(B, _gen(6), 4, H, D, block)
    plain = _clone(B, C)
    B.kv8_append(plain, k.cuda(), v.cuda(), slots.cuda())
    B.kv8_append_rotary(C, k.cuda(), v.cuda(), slots.cuda(), torch.zeros((T,), dtype=torch.int32).cuda(), _angles(B, 48, interleaved))
    assert _same(C, plain)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rotary_with_numbers_that_are_not_finite(B, interleaved):
    """A NaN turns its pair into NaN, stored as 0, and does not count for the scale; other numbers are stored as without it."""
    g, H, D, block = _gen(7), 2, 64, 16
    slots, positions = _runs(g, block, [(1, 0, 16, False), (0, 0, 3, False)]), torch.arange(19, dtype=torch.int32) + 5
    k, v = (torch.randn((19, H, D), generator=g).half() for _ in range(2))
    k[2, 1, 3] = 0.001
    k[2, 1, 2 if interleaved else 3 + 32] = 0.001
    angles = _angles(B, 32, interleaved)
    clean, C = (B.KVCache8.new(2, H, D, block) for _ in range(2))
    B.kv8_append_rotary(clean, k.cuda(), v.cuda(), slots.cuda(), positions.cuda(), angles)
    k[2, 1, 3] = float("nan")
    B.kv8_append_rotary(C, k.cuda(), v.cuda(), slots.cuda(), positions.cuda(), angles)
    want = clean.k.clone()
    want[1, 1, 2, 3] = want[1, 1, 2, 2 if interleaved else 3 + 32] = 0
    assert torch.equal(C.k, want) and torch.equal(C.k_scale, clean.k_scale) and torch.equal(C.v, clean.v)


@pytest.mark.parametrize("T,tile", [(512, 1), (513, 16), (1300, 16)])
def test_append_rotary_on_both_sides_of_its_tiles(B, T, tile):
    """One token at a time and tiles of sixteen store the same: the keys turned by hand would be rounded in between, so against a call per block."""
    g, H, D, block = _gen(8), 2, 128, 16
    blocks = -(-T // block)
    order = torch.randperm(blocks, generator=g)
    slots = torch.cat([order[i] * block + torch.arange(min(block, T - i * block)) for i in range(blocks)]).int().cuda()
    positions = (torch.arange(T, dtype=torch.int32) + 77).cuda()
    k, v, q = (torch.randn((T, n, D), generator=g).bfloat16().cuda() for n in (H, H, 3))
    angles = _angles(B, 64, False)
    one, many = B.KVCache8.new(blocks, H, D, block), B.KVCache8.new(blocks, H, D, block)
    got = B.kv8_append_rotary(one, k, v, slots, positions, angles, q)
    for a in range(0, T, 160):
        b = min(a + 160, T)
        B.kv8_append_rotary(many, k[a:b], v[a:b], slots[a:b].contiguous(), positions[a:b].contiguous(), angles)
    assert _same(one, many) and torch.equal(got, B.rotary(q, positions, angles))


@pytest.mark.parametrize("T", [700, 4500])
@pytest.mark.parametrize("D,block,H", [(64, 128, 3), (96, 64, 3), (128, 32, 5), (256, 16, 3), (256, 128, 1)])
def test_append_rotary_of_runs_that_waves_share(B, D, block, H, T):
    """A prompt in two parts that meet inside a block, whose scale the second one raises: rows that do not turn are stored as w4a4_kv8_append stores them, numbers
    that are not finite among them, and rows that turn as a call for each block stores them."""
    g, t = _gen(D + block), torch.float16
    blocks, half = -(-T // block) + 1, T // 2 + 3
    order = torch.randperm(blocks, generator=g)
    at = torch.arange(T) + 5
    slots = (order[at // block] * block + at % block).int()
    k, v = ((torch.randn((T, H, D), generator=g) * torch.where(torch.arange(T) < half, 1, 8)[:, None, None]).to(t) for _ in range(2))
    still, C = torch.full((T,), -1, dtype=torch.int32).cuda(), _cache(B, g, blocks, H, D, block)
    plain, angles, parts = _clone(B, C), _angles(B, D // 2, False), ((0, half), (half, T))
    odd_k, odd_v = k.clone(), v.clone()
    odd_k[3, 0, 1], odd_k[half + 40, H - 1, D - 1], odd_v[17, H - 1, 2], odd_v[T - 1, 0, 0] = float("nan"), float("inf"), -float("inf"), float("nan")
    for lo, hi in parts:
        B.kv8_append(plain, odd_k[lo:hi].cuda(), odd_v[lo:hi].cuda(), slots[lo:hi].cuda())
        B.kv8_append_rotary(C, odd_k[lo:hi].cuda(), odd_v[lo:hi].cuda(), slots[lo:hi].cuda(), still[lo:hi], angles)
        assert _same(C, plain)
    positions = (torch.arange(T, dtype=torch.int32) + 1000).cuda()
    C = _cache(B, _gen(1), blocks, H, D, block)
    by_block = _clone(B, C)
    for lo, hi in parts:
        B.kv8_append_rotary(C, k[lo:hi].cuda(), v[lo:hi].cuda(), slots[lo:hi].cuda(), positions[lo:hi], angles)
        edges = [lo] + [i for i in range(lo + 1, hi) if (i + 5) % block == 0] + [hi]
        for a, b in zip(edges, edges[1:]):
            B.kv8_append_rotary(by_block, k[a:b].cuda(), v[a:b].cuda(), slots[a:b].cuda(), positions[a:b], angles)
    assert _same(C, by_block)


def test_append_rotary_of_a_last_token_behind_a_long_run(B):
    """A workgroup goes on from a run of several steps to one whose window of angles is the last token alone."""
    g, H, D, block = _gen(11), 4, 64, 64
    sizes = [64] * 65 + [6, 41, 1]                                # tokens of each block: those from 66 * 63 on are one workgroup's
    T = sum(sizes)
    assert T >= 4096 and T - 42 >= 66 * 63 and T <= 67 * 63
    slots = torch.cat([b * block + torch.arange(n) for b, n in enumerate(sizes)]).int()
    positions = torch.randint(0, 5000, (T,), generator=g).int().cuda()
    k, v = (torch.randn((T, H, D), generator=g).half().cuda() for _ in range(2))
    angles = _angles(B, 32, False)
    once, by_block = (B.KVCache8.new(len(sizes), H, D, block) for _ in range(2))
    B.kv8_append_rotary(once, k, v, slots.cuda(), positions, angles)
    a = 0
    for n in sizes:
        B.kv8_append_rotary(by_block, k[a:a + n], v[a:a + n], slots[a:a + n].cuda(), positions[a:a + n], angles)
        a += n
    for b, n in enumerate(sizes):                                 # (what lies behind a block's tokens means nothing)
        assert torch.equal(once.k[b, :, :n], by_block.k[b, :, :n]) and torch.equal(once.v[b, :, :, :n], by_block.v[b, :, :, :n])
    assert torch.equal(once.k_scale, by_block.k_scale) and torch.equal(once.v_scale, by_block.v_scale)


def test_captured_and_replayed(B):
    g, H, G, D, block, T = _gen(9), 2, 6, 64, 16, 30
    angles = _angles(B, 32, True)
    q, k, v = (torch.randn((T, n, D), generator=g).half().cuda() for n in (G, H, H))
    slots, positions = torch.arange(T, dtype=torch.int32).cuda(), torch.arange(T, dtype=torch.int32).cuda()
    C = B.KVCache8.new(2, H, D, block)
    calls = [B.PreparedKV8AppendRotary(C, k, v, slots, positions, angles, q), B.PreparedRotary(q, positions, angles, inverse=True)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for call in calls:
            call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in calls:
            call()
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g).half())
        positions.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        eager = B.KVCache8.new(2, H, D, block)
        assert torch.equal(calls[0].q, B.kv8_append_rotary(eager, k, v, slots, positions, angles, q)) and _same(C, eager)
        assert torch.equal(calls[1].out, B.rotary(q, positions, angles, inverse=True))


def test_nothing_to_do(B):
    angles, e = _angles(B, 32, False), torch.empty((0,), dtype=torch.int32, device="cuda")
    C = B.KVCache8.new(1, 2, 64)
    none = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    assert B.rotary(none, e, angles).shape == (0, 2, 64) and B.kv8_append_rotary(C, none, none, e, e, angles, none).shape == (0, 2, 64)
    assert not C.k.any() and not C.k_scale.any()
