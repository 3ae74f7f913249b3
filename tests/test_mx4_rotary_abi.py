"""Rotary positions and microscaled 4-bit floating point through the C ABI without a GPU: what their entry points refuse, and what they accept as nothing to do."""
import ctypes
import os

import pytest

P = 0x1000                                                        # an address that is never read
BIG = 0x7FFFFFFF


@pytest.fixture(scope="module")
def b():
    from paper_2301_12017_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2301_12017_amd import build
        build.build(verbose=False)
    return binding


def _mx4(b, rows=8, K=64, q=P, scale=P):
    return b._MX4(q, scale, rows, K)


def _bad_operands(b):
    return ([(_mx4(b, **kw), -1) for kw in ({"rows": -1}, {"K": 0}, {"K": -32}, {"q": None}, {"scale": None})] +
            [(_mx4(b, **kw), -2) for kw in ({"K": 48}, {"K": 33}, {"K": (1 << 30) + 32}, {"q": P + 8}, {"scale": P + 2})])


def test_mx4_quantize_and_dequantize_refusals(b):
    L = b.lib()

    def quantize(c=None, X=P, dtype=0, ldx=64):
        return L.w4a4_mx4_quantize(X, dtype, ldx, ctypes.byref(c or _mx4(b)), None)

    def dequantize(c=None, dtype=0, X=P):
        return L.w4a4_mx4_dequantize(ctypes.byref(c or _mx4(b)), dtype, X, None)

    assert L.w4a4_mx4_quantize(P, 0, 64, None, None) == -1 and L.w4a4_mx4_dequantize(None, 0, P, None) == -1
    for c, rc in _bad_operands(b):
        assert quantize(c) == rc and dequantize(c) == rc
    assert quantize(dtype=2) == -1 and quantize(ldx=56) == -1 and quantize(X=None) == -1 and quantize(ldx=68) == -2 and quantize(X=P + 8) == -2
    assert dequantize(dtype=-1) == -1 and dequantize(X=None) == -1 and dequantize(X=P + 4) == -2
    assert quantize(_mx4(b, rows=0), X=None) == 0 and dequantize(_mx4(b, rows=0, q=None, scale=None), X=None) == 0
    large = _mx4(b, rows=BIG, K=32768)                            # more workgroups than a grid has
    assert quantize(large, ldx=32768) == -2 and dequantize(large) == -2
    many = _mx4(b, rows=(1 << 28) + 1, K=64)                      # a thread more than a launch counts
    assert quantize(many) == -2 and dequantize(many) == -2


def test_mx4_linear_refusals(b):
    L = b.lib()

    def f(A=None, W=None, bias=None, act=0, dtype=0, out=P):
        return L.w4a4_mx4_linear(ctypes.byref(A or _mx4(b, rows=4)), ctypes.byref(W or _mx4(b)), bias, act, dtype, out, None)

    assert L.w4a4_mx4_linear(None, ctypes.byref(_mx4(b)), None, 0, 0, P, None) == -1 and L.w4a4_mx4_linear(ctypes.byref(_mx4(b)), None, None, 0, 0, P, None) == -1
    for c, rc in _bad_operands(b):
        assert f(A=c) == rc and f(W=c) == rc
    assert f(W=_mx4(b, K=96)) == -1 and f(W=_mx4(b, rows=0)) == -1 and f(act=2) == -1 and f(dtype=3) == -1 and f(out=None) == -1
    assert f(W=_mx4(b, rows=12)) == -2 and f(out=P + 8) == -2 and f(bias=P + 2) == -2
    assert f(A=_mx4(b, rows=BIG), W=_mx4(b, rows=BIG - 7)) == -2      # more tiles than a grid has
    assert f(A=_mx4(b, rows=0), out=None) == 0


def test_mx4_linear_a16_refusals(b):
    L = b.lib()

    def f(X=P, dtype=0, M=4, ldx=64, W=None, bias=None, act=0, out=P):
        return L.w4a4_mx4_linear_a16(X, dtype, M, ldx, ctypes.byref(W or _mx4(b)), bias, act, out, None)

    assert L.w4a4_mx4_linear_a16(P, 0, 4, 64, None, None, 0, P, None) == -1
    for c, rc in _bad_operands(b):
        assert f(W=c) == rc
    assert f(M=-1) == -1 and f(ldx=56) == -1 and f(dtype=2) == -1 and f(act=-1) == -1 and f(W=_mx4(b, rows=0)) == -1 and f(X=None) == -1 and f(out=None) == -1
    assert f(W=_mx4(b, rows=12)) == -2 and f(ldx=68) == -2 and f(X=P + 4) == -2 and f(out=P + 8) == -2 and f(bias=P + 4) == -2
    assert f(M=BIG, W=_mx4(b, rows=BIG - 7)) == -2 and f(ldx=1 << 24) == -2
    assert f(M=0, X=None, out=None) == 0


def _angles(b, turns=P, pairs=32, interleaved=0, magnitude=1.0, inverse=0):
    return b._RotaryAngles(turns, pairs, interleaved, magnitude, inverse)


def _bad_angles(b):
    return [(_angles(b, **kw), rc) for kw, rc in (({"turns": None}, -1), ({"pairs": 0}, -1), ({"pairs": -1}, -1), ({"pairs": 33}, -1), ({"interleaved": 2}, -1), ({"inverse": -1}, -1),
                                                  ({"magnitude": 0.0}, -1), ({"magnitude": -1.0}, -1), ({"magnitude": float("nan")}, -1), ({"magnitude": float("inf")}, -1), ({"turns": P + 4}, -2))]


def test_rotary_refusals(b):
    L = b.lib()

    def f(X=P, dtype=0, tokens=4, heads=2, features=64, ldx=128, positions=P, R=None, out=2 * P, ldo=128):
        return L.w4a4_rotary(X, dtype, tokens, heads, features, ldx, positions, ctypes.byref(R or _angles(b)), out, ldo, None)

    assert L.w4a4_rotary(P, 0, 4, 2, 64, 128, P, None, 2 * P, 128, None) == -1
    for r, rc in _bad_angles(b):
        assert f(R=r) == rc
    assert f(tokens=-1) == -1 and f(heads=0) == -1 and f(features=0) == -1 and f(dtype=2) == -1 and f(ldx=120) == -1 and f(ldo=64) == -1
    assert f(X=None) == -1 and f(out=None) == -1 and f(positions=None) == -1 and f(out=P, ldo=136) == -1
    assert f(features=68, ldx=136, ldo=136) == -2 and f(features=264, ldx=528, ldo=528) == -2 and f(ldx=132) == -2 and f(ldo=130) == -2 and f(X=P + 2) == -2 and f(out=P + 8) == -2
    assert f(heads=BIG, features=256) == -1
    assert f(tokens=(1 << 28) + 1, heads=16, features=128, ldx=2048, ldo=2048, R=_angles(b, interleaved=1)) == -2      # more threads than a launch counts
    assert f(tokens=0, X=None, out=None, positions=None) == 0


def test_kv8_append_rotary_refusals(b):
    L = b.lib()

    def f(c=None, R=None, **kw):
        d = dict(k=P, v=P, q=P, q_out=2 * P, slots=P, positions=P, dtype=0, tokens=4, ldk=128, ldv=128, heads=4, ldq=256)
        d.update(kw)
        return L.w4a4_kv8_append_rotary(ctypes.byref(c or b._KV8Cache(P, P, P, P, 4, 2, 16, 64)), ctypes.byref(b._KV8Rows(**d)), ctypes.byref(R or _angles(b)), None)

    cache, rows = b._KV8Cache(P, P, P, P, 4, 2, 16, 64), b._KV8Rows(P, P, None, None, P, P, 0, 0, 128, 128, 0, 0)
    assert L.w4a4_kv8_append_rotary(None, ctypes.byref(rows), ctypes.byref(_angles(b)), None) == -1
    assert L.w4a4_kv8_append_rotary(ctypes.byref(cache), None, ctypes.byref(_angles(b)), None) == -1
    assert L.w4a4_kv8_append_rotary(ctypes.byref(cache), ctypes.byref(rows), None, None) == -1
    assert L.w4a4_kv8_append_rotary(ctypes.byref(cache), ctypes.byref(rows), ctypes.byref(_angles(b)), None) == 0
    for r, rc in _bad_angles(b):
        assert f(R=r) == rc
    assert f(c=b._KV8Cache(P, P, P, P, 4, 2, 24, 64)) == -2 and f(c=b._KV8Cache(P, P, P, P, 4, 2, 16, 80)) == -2 and f(c=b._KV8Cache(None, P, P, P, 4, 2, 16, 64)) == -1
    for kw in ({"tokens": -1}, {"dtype": 2}, {"ldk": 120}, {"ldv": 64}, {"k": None}, {"v": None}, {"slots": None}, {"positions": None}, {"q_out": None}, {"q": None}, {"q_out": P},
               {"heads": 0}, {"ldq": 248}):
        assert f(**kw) == -1, kw
    for kw in ({"ldk": 132}, {"ldv": 132}, {"k": P + 8}, {"v": P + 2}, {"ldq": 260}, {"q": P + 8}, {"q_out": P + 4}):
        assert f(**kw) == -2, kw
    assert f(tokens=0) == 0 and f(tokens=0, k=None, positions=None) == 0
    assert f(tokens=1 << 28) == -2 and f(tokens=BIG, q=None, q_out=None) == -2       # more threads than a launch counts


def test_calls_laid_out_once_reach_their_entry_point(b):
    L, at = b.lib(), ctypes.addressof
    Q, R = _mx4(b), _angles(b)

    def run(entry, pointers, ints=()):
        call = b._Call((ctypes.c_void_p * 10)(*pointers), 0, (ctypes.c_int * 6)(*ints), 0.0, entry)
        return L.w4a4_run_call(ctypes.byref(call), None)

    names = b._Prepared.ENTRIES
    assert names[11:] == ("w4a4_rotary", "w4a4_kv8_append_rotary", "w4a4_mx4_quantize", "w4a4_mx4_dequantize", "w4a4_mx4_linear", "w4a4_mx4_linear_a16")
    assert run(11, (P, P, at(R), 2 * P), (0, 0, 2, 64, 128, 128)) == 0 and run(11, (P, P, at(R), 2 * P), (0, 4, 2, 64, 128, 120)) == -1 and run(11, (P, P, at(R), 2 * P), (0, 4, 2, 64, 132, 128)) == -2
    assert run(12, (P, None, at(R))) == -1
    assert run(13, (P, at(Q)), (0, 56)) == -1 and run(13, (P, at(Q)), (0, 68)) == -2 and run(14, (at(Q), P), (2,)) == -1 and run(14, (at(Q), P + 4), (0,)) == -2
    assert run(15, (at(Q), at(Q), None, P), (2, 0)) == -1 and run(15, (at(Q), at(Q), None, P + 8), (0, 1)) == -2
    assert run(16, (P, at(Q), None, P), (0, 4, 56, 0)) == -1 and run(16, (P, at(Q), None, P), (0, 0, 64, 0)) == 0 and run(16, (P, at(Q), None, P), (0, 4, 72, 2)) == -1
    assert run(17, (P, P, P, P)) == -1


def test_binding_refuses_what_does_not_fit(b):
    import torch
    q, s = torch.zeros((1, 8, 64), dtype=torch.uint8), torch.zeros((1, 8), dtype=torch.int32)
    for args in ((q, s, 64), (q, s, 160), (q, s, 48)):            # in host memory; other planes than K has; no multiple of 32
        with pytest.raises(AssertionError):
            b.MX4(*args)
    with pytest.raises(AssertionError):
        b.MX4.from_rows(torch.zeros((4, 24), dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.uint8))
    angles = b.RotaryAngles([1.0, 0.5], device="cpu")
    with pytest.raises(AssertionError):
        b.rotary(torch.zeros((1, 1, 8), dtype=torch.float16), torch.zeros(1, dtype=torch.int32), angles)


def test_decoder_refuses_what_it_cannot_place_or_name(b):
    import torch
    from paper_2301_12017_amd import decoder as dec
    books = dec.Books(3, 64, 12, 16, device="cpu")
    layer = type("Layer", (), {"angles": None})()
    with pytest.raises(ValueError):                               # no table of positions, and nothing that turns
        dec.Decoder([layer], torch.zeros((8, 64), dtype=torch.float16), None, books)
    with pytest.raises(ValueError):
        dec.quantized(torch.zeros((8, 64), dtype=torch.float16), "int3")
