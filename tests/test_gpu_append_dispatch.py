"""The append with positions on both sides of every border of its dispatch: tokens of a workgroup (1 up to 512 tokens, a 128th of them up to 2047, 16, from 4096 on as many as a block
has, 63 at most), and waves that share a run (where a workgroup has one token, only up to 2048 tokens times heads times waves)."""
import pytest
import torch

from tests.gpu_util import has_gpu
from tests.test_gpu_rotary import _cache, _clone, _gen, _same

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.fixture(scope="module")
def B():
    from paper_2301_12017_amd import binding
    binding.lib()
    return binding


def _lengths(kind, T, block, g):
    """Tokens of each run, T in all."""
    n, left = [], T
    while left:
        long = {"single": False, "prompts": True}.get(kind)
        if long is None:
            long = torch.rand((), generator=g) < 0.4
        n.append(min(left, (block if torch.rand((), generator=g) < 0.7 else int(torch.randint(1, block + 1, (), generator=g))) if long else 1))
        left -= n[-1]
    return n


def _check(B, T, D, H, block, kind, interleaved=False):
    """One call against a call for each run: the same bits, whatever their workgroups; and rows that do not turn against the append without positions.  Scales that rise and
    blocks that begin anew, slots in order and not, tokens that are not stored, numbers that are not finite."""
    g = _gen(T + D + block)
    lengths = _lengths(kind, T, block, g)
    order, slots, edges = torch.randperm(len(lengths), generator=g), [], [0]
    for b, n in zip(order.tolist(), lengths):
        at = torch.arange(n) + int(torch.randint(0, block - n + 1, (), generator=g))
        if torch.rand((), generator=g) < 0.2:
            at = at[torch.randperm(n, generator=g)]
        slots += [-1] * n if torch.rand((), generator=g) < 0.1 else (b * block + at).tolist()
        edges.append(edges[-1] + n)
    slots = torch.tensor(slots, dtype=torch.int32).cuda()
    size = torch.exp(torch.randn((T, 1, 1), generator=g))
    k, v, q = ((torch.randn((T, n, D), generator=g) * size).half() for n in (H, H, 2 * H))
    for i in torch.randint(0, T, (12,), generator=g).tolist():
        k[i, i % H, i % D], v[T - 1 - i, i % H, (7 * i) % D] = (float("nan"), float("inf"), -float("inf"))[i % 3], (float("inf"), float("nan"), -float("inf"))[i % 3]
    k, v, q = k.cuda(), v.cuda(), q.cuda()
    positions = torch.randint(0, 100000, (T,), generator=g).int()
    positions[::11] = -1
    positions, still = positions.cuda(), torch.full((T,), -1, dtype=torch.int32).cuda()
    angles = B.RotaryAngles(B.rotary_frequencies(D // 2)[0], interleaved)
    start = _cache(B, g, len(lengths), H, D, block)
    once, apart, plain, turned = (_clone(B, start) for _ in range(4))
    got = B.kv8_append_rotary(once, k, v, slots, positions, angles, q)
    for a, b in zip(edges, edges[1:]):
        B.kv8_append_rotary(apart, k[a:b], v[a:b], slots[a:b].clone(), positions[a:b].clone(), angles)
    stored = bool((slots >= 0).any())                             # (of a single run that is not stored there is nothing)
    assert _same(once, apart) and _same(once, start) != stored
    assert torch.equal(got, B.rotary(q, positions, angles))
    B.kv8_append(plain, k, v, slots)
    B.kv8_append_rotary(turned, k, v, slots, still, angles)
    assert _same(plain, turned)


@pytest.mark.parametrize("kind", ["single", "prompts", "mixed"])
@pytest.mark.parametrize("block", [16, 64, 128])
@pytest.mark.parametrize("T", [511, 512, 513, 640, 1023, 2047, 2048, 3000, 4095, 4096])
def test_tokens_of_a_workgroup(B, T, block, kind):
    _check(B, T, 128, 2, block, kind)


@pytest.mark.parametrize("kind", ["prompts", "mixed"])
@pytest.mark.parametrize("T,H", [(400, 8), (511, 5), (128, 8), (129, 8), (300, 3), (64, 8), (65, 9)])
@pytest.mark.parametrize("D,block", [(64, 32), (128, 128), (96, 32), (256, 16), (256, 128)])
def test_waves_that_share_a_run_or_do_not(B, D, block, T, H, kind):
    _check(B, T, D, H, block, kind, interleaved=D == 96)


@pytest.mark.parametrize("D,block,H", [(64, 128, 3), (96, 64, 3), (256, 32, 1), (256, 128, 3)])
@pytest.mark.parametrize("T", [700, 2048, 4096, 5000])
def test_other_heads(B, D, block, H, T):
    _check(B, T, D, H, block, "mixed", interleaved=D == 64)
