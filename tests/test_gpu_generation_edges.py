"""Token generation on the GPU where it can go wrong: rows of NaN, infinities, scales far apart, sizes at their limits, single rows of wider
arrays, shared workspaces.  Oracles and tolerances as in test_gpu_generation.py."""
import math

import pytest
import torch

from tests.gpu_util import has_gpu
from tests.test_gpu_generation import TYPES, U, B, _attention_case, _gen, _random_cache, _weight  # noqa: F401 (B is a fixture)

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


# Queries, keys, window, features: few rows of a request and head, many.
FAR_FEW = [(1, 100, 0, 64), (5, 99, 0, 128), (5, 291, 40, 64), (16, 3000, 0, 128), (3, 200, 0, 256)]
FAR_MANY = [(40, 100, 0, 64), (70, 130, 0, 128), (300, 900, 0, 128), (40, 600, 17, 96), (100, 300, 0, 256), (40, 20000, 0, 64)]
# Scale of one block of values, factor of the others' (0.015 to 0.03), types.
FAR_SCALES = [(2.0 ** -30, 2.0 ** -60, "fp16"), (2.0 ** -30, 2.0 ** -60, "bf16"), (1.0, 2.0 ** -3, "fp16"), (1.0, 2.0 ** -3, "bf16"), (2.0 ** 9, 2.0 ** -24, "fp16"), (2.0 ** 9, 2.0 ** -24, "bf16"),
              (2.0 ** 100, 2.0 ** -3, "bf16"), (2.0 ** -70, 2.0 ** -90, "bf16")]


def _far_case(B, n, keys, window, D, most, others, dtype, kept):
    """kept: log2 of the products, relative to a row's largest, below which weights lose bits."""
    H, block, g, t = 2, 16, _gen(n + keys), TYPES[dtype]
    blocks = -(-keys // block)
    cache = _random_cache(B, g, blocks, H, block, D)
    cache.v_scale.mul_(others)
    far = (keys - 1) // block - (1 if n > 20 else 0)
    cache.v_scale[far] = most
    if most >= 1:                                                 # its keys are opposite to the queries: rows that see them look elsewhere
        cache.k[far] = -60
        cache.k_scale[far] = 0.02
    q = (torch.randn((n, 2 * H, D), generator=g) * 0.3 + 1.0).to(t)
    start, lens = torch.tensor([0, n], dtype=torch.int32), torch.tensor([keys], dtype=torch.int32)
    out, lse = (x.cpu().double() for x in B.kv8_attention(q.cuda(), cache, torch.arange(blocks, dtype=torch.int32, device="cuda")[None], lens.cuda(), start.cuda(), n, keys,
                                                          D ** -0.5, window=window, want_lse=True))
    K = (cache.k.cpu().double() * cache.k_scale.cpu().double()[:, :, None, None]).permute(1, 0, 2, 3).reshape(H, -1, D)[:, :keys]
    V = (cache.v.cpu().double() * cache.v_scale.cpu().double()[:, :, None, None]).permute(1, 0, 3, 2).reshape(H, -1, D)[:, :keys]
    vs = cache.v_scale.cpu().double().t().repeat_interleave(block, 1)[:, :keys]
    at, key = keys - n + torch.arange(n)[:, None], torch.arange(keys)[None]
    sees = (key <= at) & (key > at - window if window else key >= 0)
    h, tiny = torch.finfo(t).eps / 2, torch.finfo(t).smallest_normal * torch.finfo(t).eps
    for head in range(2 * H):
        x = q[:, head].double() @ K[head // 2].t() * D ** -0.5
        noise = (q[:, head].double().abs() @ K[head // 2].abs().t() * D ** -0.5).amax(1, keepdim=True)
        x = torch.where(sees, x, -math.inf)
        z = torch.logsumexp(x, 1, keepdim=True)
        p = torch.exp(x - z)
        y, size = p @ V[head // 2], p @ V[head // 2].abs()
        # a score: D + 6 roundings of its terms' sum, three of numbers below 2^8 when the exponent of a scale comes in (each half a step of 2^-16 and the log
        # of 2: 92 U); a weight: that, the exponential and half a step of fp16; sums: a rounding per instruction, under the row's OWN sizes
        weight = (D + 6) * U * noise + 300 * U + 2.0 ** -22
        # a product of weight and scale below 2^kept of the row's largest: half a step of fp16's subnormal numbers (2^-11 of the smallest normal one) for each key
        largest = (p * vs[head // 2]).amax(1, keepdim=True) * 127
        tol = size * (2.0 ** -11 + 2 * weight + (keys / 32 + 40) * U) + h * y.abs() * (1 + 2.0 ** -10) + tiny + keys * 2.0 ** (kept - 11) * largest
        assert torch.all((out[:, head] - y).abs() <= tol), (head, float(((out[:, head] - y).abs() / tol).max()))
        assert torch.all((lse[:, head, None] - z).abs() <= weight + (keys / 16 + keys / 32 + 40) * U + 2.0 ** -22 * (1 + z.abs()))


@pytest.mark.parametrize("most, others, dtype", FAR_SCALES)
@pytest.mark.parametrize("n, keys, window, D", FAR_FEW)
def test_values_behind_a_far_larger_scale_keep_their_bits(B, n, keys, window, D, most, others, dtype):
    """Rows that do not see the block of the largest scale, and rows that give its keys hardly any weight, come out as exactly as they would without it."""
    _far_case(B, n, keys, window, D, most, others, dtype, -27)


@pytest.mark.parametrize("most, others, dtype", [(min(most, 2.0 ** 80), others, dtype) for most, others, dtype in FAR_SCALES])
@pytest.mark.parametrize("n, keys, window, D", FAR_MANY)
def test_values_behind_a_far_larger_scale_keep_their_bits_in_prompts(B, n, keys, window, D, most, others, dtype):
    _far_case(B, n, keys, window, D, most, others, dtype, -20)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K,group,asym", [(7, 264, 512, 128, True), (7, 256, 768, 0, False), (20, 72, 320, 64, True), (40, 136, 384, 128, False), (9, 40, 96, 32, False), (70, 8200, 256, 0, True)])
def test_linear_w4a16_of_infinities(B, M, N, K, group, asym, dtype):
    """Infinities of one sign, of both, NaN, and (bf16) numbers that pass fp32 with the offset of the codes: what the definition has, in those rows alone."""
    g, t = _gen(M + N), TYPES[dtype]
    W, c, scale, zero = _weight(B, g, N, K, group, asym)
    X = torch.randn((M, K), generator=g).to(t)
    inf, nan = float("inf"), float("nan")
    X[0, 5] = inf
    X[1, K - 1] = -inf
    X[2, 3], X[2, K // 2] = inf, -inf
    X[3, 7] = nan
    X[4, :9] = inf
    if dtype == "bf16":
        X[6, 2], X[6, 40] = 1e37, 3e36
    got = B.linear_w4a16(X.cuda(), W).cpu().double()
    w = (c.view(N, -1, group or K) * scale.double()[:, :, None] + (0 if zero is None else zero.double()[:, :, None])).view(N, K)
    y = torch.stack([(w * x).sum(1) for x in X.double()])         # (0 times an infinity is NaN here)
    assert bool(torch.isinf(y[:2]).any()) and (asym or bool(torch.isnan(y[:2]).any())) and bool(torch.isnan(y[2]).any()) and bool(torch.isnan(y[3]).all()) and bool(torch.isfinite(y[5:]).all())
    assert torch.equal(torch.isnan(got), torch.isnan(y)) and torch.equal(got[torch.isinf(y)], y[torch.isinf(y)]) and torch.equal(torch.isinf(got), torch.isinf(y))
    rows = torch.isfinite(X.double()).all(1)
    off = 136 if dtype == "bf16" else 8
    size = X.double()[rows].abs() @ (w.abs() + off * scale.double().amax()).t()
    h = torch.finfo(t).eps / 2
    # sums with the codes' offset in them, or one after the other: K + 4 roundings at most
    assert torch.all((got[rows] - y[rows]).abs() <= h * y[rows].abs() * (1 + 1e-5) + (K + 4) * U * size + 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_linear_w4a16_gelu_of_nan_of_either_sign(B, dtype):
    g, t = _gen(1), TYPES[dtype]
    W, *_ = _weight(B, g, 40, 256, 128, False)
    X = torch.randn((5, 256), generator=g).to(t)
    want = B.linear_w4a16(X.cuda(), W, None, B.ACT_GELU)
    bits = X.view(torch.int16)
    bits[1, 9], bits[3, 200] = (0x7E00, 0x7E00 - 0x8000) if dtype == "fp16" else (0x7FC0, 0x7FC0 - 0x8000)
    X[4, 0], X[4, 1] = float("inf"), -float("inf")
    got = B.linear_w4a16(X.cuda(), W, None, B.ACT_GELU)
    assert torch.isnan(got[[1, 3]]).all() and torch.equal(got[[0, 2]], want[[0, 2]])
    assert torch.equal(torch.isnan(got[4]), torch.isnan(B.linear_w4a16(X.cuda(), W)[4]))


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30 + 1, 2 ** 30])
@pytest.mark.parametrize("n, lens", [([5, 1], [2, 70]), ([70, 9], [50, 9])])
def test_kv8_attention_with_the_largest_windows(B, n, lens, window):
    """More queries than keys, so that the first ones stand at negative positions."""
    _attention_case(B, n, lens, 1, 2, 64, 16, window, "fp16", seed=n[0])


@pytest.mark.parametrize("block", [16, 128])
def test_kv8_plan_makes_no_slot_of_what_is_no_block(B, block):
    """Entries of a table and of a ring whose number, times the tokens of a block, passes 32 bits."""
    wild = [2 ** 32 // block + 5, -5, 2 ** 31 - 1, -2 ** 31, 2 ** 31 // block, 2 ** 31 // block - 1, 3]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    R = len(wild)
    call = B.kv8_plan(i32([3] * R), i32([2] * R), i32([[w, 9] for w in wild]), i32([7]), i32([0, 0]), block, 2 * R)
    want = [s for w in wild for s in ([block * w + 3, block * w + 4] if 0 <= w < 2 ** 31 // block else [-1, -1])]
    assert call.slots.tolist() == want and call.positions.tolist() == [3, 4] * R
    call = B.kv8_plan(i32([0] * R), i32([1] * R), i32([[9, 9]] * R), i32(wild), i32([0, R]), block, R)
    assert call.slots.tolist() == [block * w if 0 <= w < 2 ** 31 // block else -1 for w in wild] and call.positions.tolist() == [0] * R
    assert call.table[:, 0].tolist() == wild


@pytest.mark.parametrize("stride", [1001, 3, 64 * 4])
def test_single_rows_of_any_stride(B, stride):
    """One row of a wider array, or of a broadcast one: its stride says nothing."""
    g = _gen(stride)
    row = torch.randn((1, 256), generator=g).half().cuda()
    x = row.as_strided((1, 256), (stride, 1))
    W, *_ = _weight(B, g, 64, 256, 64, True)
    assert torch.equal(B.linear_w4a16(x, W), B.linear_w4a16(row.clone(), W))
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    found = []
    for kv in (row.view(1, 4, 64), row.as_strided((1, 4, 64), (stride, 64, 1))):
        cache = B.KVCache8.new(2, 4, 64)
        B.kv8_append(cache, kv, kv, i32(16))
        found.append((cache.k, cache.v, B.kv8_attention(kv, cache, i32(1)[None], i32(1), i32(0, 1), 1, 1, 0.125)))
    assert all(torch.equal(a, b) for a, b in zip(*found)) and found[0][0].any()


def test_generation_refuses_host_tensors(B):
    """A result, a bias or weights that are not on the GPU are refused before anything is launched."""
    g = _gen(1)
    W, *_ = _weight(B, g, 64, 256, 64, False)
    x = torch.randn((3, 256), generator=g).half().cuda()
    host = B.QWeight(W.q.cpu(), W.scale.cpu(), None, None, None, 64, 256, 64, B.SYM)
    for args in ((x, W, torch.zeros(64, dtype=torch.float16)), (x, W, None, B.ACT_NONE, torch.zeros((3, 64), dtype=torch.float16)), (x, host), (x.cpu(), W)):
        with pytest.raises(AssertionError):
            B.PreparedLinearW4A16(*args)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache = B.KVCache8.new(2, 4, 64)
    with pytest.raises(AssertionError):
        B.PreparedKV8Attention(x.view(3, 4, 64), cache, i32(1)[None], i32(3), i32(0, 3), 3, 3, 0.125, out=torch.zeros((3, 4, 64), dtype=torch.float16))


def test_one_workspace_for_calls_of_every_shape(B):
    """Cut requests, batches that mix prompts and single tokens, prompts, smaller and larger in turn: the bits of calls with workspaces of their own."""
    g, shared = _gen(3), B.KV8Workspace()
    cache = _random_cache(B, g, 700, 2, 32, 128)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    shapes = [([1], [9000]), ([1, 40, 1, 3, 100], [700, 60, 2900, 300, 4000]), ([1] * 9, [2000] * 9), ([700], [5000]), ([2, 1], [6000, 3]), ([1], [30]), ([400, 90], [3000, 2000])]
    calls, want = [], []
    for n, lens in shapes:
        have = [-(-x // 32) for x in lens]
        table = torch.zeros((len(n), max(have)), dtype=torch.int32)
        ids = torch.randperm(700, generator=g).int()
        for r, h in enumerate(have):
            table[r, :h] = ids[sum(have[:r]):sum(have[:r + 1])]
        args = (torch.randn((sum(n), 8, 128), generator=g).half().cuda(), cache, table.cuda(), i32(lens), i32([sum(n[:i]) for i in range(len(n) + 1)]), max(n), max(lens), 0.09)
        want.append([t.clone() for t in B.kv8_attention(*args, want_lse=True)])
        calls.append(args)
    for _ in range(2):
        for args, w in zip(calls, want):
            got = B.kv8_attention(*args, want_lse=True, workspace=shared)
            assert all(torch.equal(a, b) for a, b in zip(got, w))
    size = shared.bytes.numel()
    assert size >= 700 * 1024 and not shared.bytes[:shared.ZEROS].any()
    B.kv8_attention(*calls[0], workspace=shared)
    assert shared.bytes.numel() == size


def test_a_workspace_is_not_filled_with_zeros(B, monkeypatch):
    """Of the workspace of a prompt, a hundred megabytes, only the counters are."""
    cache = B.KVCache8.new(20, 8, 128, 32)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, q, args = torch.arange(20, dtype=torch.int32, device="cuda")[None], torch.zeros((300, 8, 128), dtype=torch.float16, device="cuda"), (i32(600), i32(0, 300))
    made, zeros, zero_ = [], torch.zeros, torch.Tensor.zero_
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: (made.append(zeros(*a, **k)), made[-1])[1])
    monkeypatch.setattr(torch.Tensor, "zero_", lambda t: (made.append(t), zero_(t))[1])
    call = B.PreparedKV8Attention(q, cache, table, *args, 300, 600, 0.09)
    call()
    assert call.workspace.numel() > 10 ** 8 and made and all(t.numel() * t.element_size() <= 18432 for t in made)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("n, keys, window, D", [(1, 100, 0, 64), (5, 99, 40, 128), (40, 100, 0, 64), (300, 900, 70, 128), (40, 200, 0, 256)])
def test_blocks_of_scale_zero_add_nothing(B, n, keys, window, D, dtype):
    """Codes under a scale of 0: rows that see no others get zeros, for the others the block's values are zeros; its keys count in the sums."""
    g, t, block = _gen(n + keys), TYPES[dtype], 16
    blocks = -(-keys // block)
    cache = _random_cache(B, g, blocks, 2, block, D)
    call = B.PreparedKV8Attention(torch.randn((n, 4, D), generator=g).to(t).cuda(), cache, torch.arange(blocks, dtype=torch.int32, device="cuda")[None],
                                  torch.tensor([keys], dtype=torch.int32, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, keys, D ** -0.5, window=window, want_lse=True)
    call()
    sums = call.lse.clone()
    kept = cache.v_scale.clone()
    for first in (0, blocks // 2, blocks):                         # blocks of scale 0: all, those before the middle and every other one behind it, every other one
        cache.v_scale.copy_(kept)
        cache.v_scale[:blocks - first] = 0
        cache.v_scale[::2] = 0
        call()
        with_codes, lse = call.out.clone(), call.lse.clone()
        held = cache.v.clone()
        cache.v[cache.v_scale[:, 0] == 0] = 0
        call()
        cache.v.copy_(held)
        # (the codes may decide a rounding of what lies in the middle between two numbers: a step)
        assert torch.equal(lse, call.lse) and torch.all((with_codes - call.out).abs().float() <= torch.finfo(t).eps * call.out.abs().float() + torch.finfo(t).smallest_normal * torch.finfo(t).eps)
        at = keys - n + torch.arange(n)
        begin = (at - window + 1).clamp(min=0) if window else at * 0
        live = [any(float(cache.v_scale[b, 0]) > 0 for b in range(int(b0) // block, int(e) // block + 1)) for b0, e in zip(begin, at)]
        none = ~torch.tensor(live).cuda()
        assert not with_codes[none].any() and (bool(none.all()) or bool(with_codes[~none].any()))
        # the sums do not depend on the scales but for their roundings: in the log a few of numbers below 2^7 and 2^-22 of the exponential
        assert torch.all((lse - sums).abs() <= 300 * U + 2.0 ** -21 + (keys / 16 + 40) * U)
