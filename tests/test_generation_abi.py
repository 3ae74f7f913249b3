"""Token generation through the C ABI without a GPU: what its entry points refuse, and what they accept as nothing to do."""
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


def test_linear_w4a16_refusals(b):
    L = b.lib()

    def f(M=4, K=64, ldx=None, N=8, group=0, mode=0, layout=0, dtype=0, act=0, x=P, o=P, bias=None, q=P, scale=P, zero=P, wk=None):
        w = b._Weight(q, scale, zero, None, N, K if wk is None else wk, group, mode, layout, None)
        return L.w4a4_linear_w4a16(x, dtype, M, K, K if ldx is None else ldx, ctypes.byref(w), bias, act, o, None)

    assert L.w4a4_linear_w4a16(P, 0, 4, 64, 64, None, None, 0, P, None) == -1
    assert f(M=-1) == -1 and f(ldx=32) == -1 and f(wk=96) == -1 and f(K=0) == -1 and f(N=0) == -1 and f(group=-32) == -1
    assert f(dtype=2) == -1 and f(act=2) == -1 and f(mode=2) == -1
    assert f(x=None) == -1 and f(o=None) == -1 and f(q=None) == -1 and f(scale=None) == -1 and f(mode=1, zero=None) == -1
    assert f(layout=1) == -2 and f(layout=2) == -2
    assert f(K=48) == -2 and f(N=12) == -2 and f(ldx=68) == -2 and f(group=48) == -2 and f(K=96, group=64) == -2
    assert f(x=P + 4) == -2 and f(o=P + 8) == -2 and f(q=P + 1) == -2 and f(bias=P + 2) == -2
    assert f(M=BIG) == -2
    assert f(M=0) == 0 and f(M=0, x=None) == 0


def test_kv8_plan_refusals(b):
    L = b.lib()

    def f(requests=4, width=8, capacity=16, block=16, tokens=4, lens=P, new=P, table=P, ring=P, state=P, so=2 * P, lo=2 * P, start=P, slots=P, pos=P):
        return L.w4a4_kv8_plan(lens, new, requests, table, width, ring, capacity, state, block, tokens, so, lo, start, slots, pos, None)

    assert f(requests=-1) == -1 and f(width=-1) == -1 and f(capacity=0) == -1 and f(block=0) == -1 and f(tokens=-1) == -1
    for name in ("lens", "new", "table", "ring", "state", "so", "lo", "start", "slots", "pos"):
        assert f(**{name: None}) == -1, name
    assert f(so=P) == -1 and f(lo=P) == -1                            # outputs in the place of inputs: the call could not be repeated
    assert f(block=8) == -2 and f(block=24) == -2 and f(block=256) == -2
    assert f(capacity=BIG) == -2                                      # slots would pass 32 bits


def _cache(b, blocks=4, heads=2, block=16, features=64, k=P, v=P, ks=P, vs=P):
    return b._KV8Cache(k, v, ks, vs, blocks, heads, block, features)


def _bad_caches(b):
    return ([(_cache(b, **kw), -1) for kw in ({"blocks": -1}, {"heads": 0}, {"block": 0}, {"features": 0}, {"k": None}, {"v": None}, {"ks": None}, {"vs": None})] +
            [(_cache(b, **kw), -2) for kw in ({"block": 8}, {"block": 48}, {"block": 256}, {"features": 32}, {"features": 80}, {"features": 512}, {"heads": 1025},
                                              {"blocks": BIG}, {"k": P + 8}, {"v": P + 4})])


def test_kv8_append_and_read_refusals(b):
    L = b.lib()

    def app(c=None, K=P, V=P, dtype=0, T=4, ldk=128, ldv=128, slots=P):
        return L.w4a4_kv8_append(ctypes.byref(c or _cache(b)), K, V, dtype, T, ldk, ldv, slots, None)

    def read(c=None, slots=P, T=4, dtype=0, K=P, V=P):
        return L.w4a4_kv8_read(ctypes.byref(c or _cache(b)), slots, T, dtype, K, V, None)

    assert L.w4a4_kv8_append(None, P, P, 0, 4, 128, 128, P, None) == -1 and L.w4a4_kv8_read(None, P, 4, 0, P, P, None) == -1
    for c, rc in _bad_caches(b):
        assert app(c) == rc and read(c) == rc
    assert app(T=-1) == -1 and app(dtype=2) == -1 and app(ldk=120) == -1 and app(ldv=64) == -1
    assert app(K=None) == -1 and app(V=None) == -1 and app(slots=None) == -1
    assert app(ldk=132) == -2 and app(ldv=130) == -2 and app(K=P + 2) == -2 and app(V=P + 8) == -2
    assert app(T=0) == 0 and app(T=0, K=None) == 0
    assert read(T=-1) == -1 and read(dtype=-1) == -1 and read(K=None) == -1 and read(V=None) == -1 and read(slots=None) == -1
    assert read(K=P + 4) == -2 and read(V=P + 8) == -2
    assert read(T=0) == 0


def test_kv8_attention_refusals(b):
    L = b.lib()

    def f(c=None, out=P, ws=None, n=0, **kw):
        d = dict(q=P, table=P, lens=P, start=P, scale=0.125, dtype=0, tokens=2, heads=4, ldq=256, requests=2, width=4, queries=1, context=64, window=0)
        d.update(kw)
        q = b._KV8Queries(**d)
        c = c or _cache(b)
        return L.w4a4_kv8_attention(ctypes.byref(c), ctypes.byref(q), out, None, ws, n, None), L.w4a4_kv8_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(q))

    assert L.w4a4_kv8_attention(None, None, P, None, None, 0, None) == -1 and L.w4a4_kv8_attention_workspace_bytes(None, None) == 0
    for c, rc in _bad_caches(b):
        assert f(c) == (rc, 0)
    for kw in ({"tokens": -1}, {"requests": -1}, {"heads": 0}, {"queries": -1}, {"context": -1}, {"window": -1}, {"width": -1}, {"dtype": 3}, {"heads": 3},
               {"ldq": 248}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}):
        assert f(**kw) == (-1, 0), kw
    for kw in ({"q": None}, {"table": None}, {"lens": None}, {"start": None}, {"out": None}):
        assert f(**kw)[0] == -1, kw
    assert f(ldq=260) == (-2, 0) and f(q=P + 8)[0] == -2 and f(out=P + 2)[0] == -2 and f(requests=70000, tokens=70000)[0] == -2
    for kw in ({"tokens": 0}, {"requests": 0}, {"queries": 0}):
        assert f(**kw) == (0, 0), kw
    # many keys and few rows: the keys are shared out, which takes a workspace
    rc, need = f(width=10000, context=150000)
    assert rc == -3 and need > 0
    assert f(width=10000, context=150000, ws=2 * P, n=need - 1)[0] == -3 and f(width=10000, context=150000, ws=2 * P + 4, n=need)[0] == -2


def test_generation_calls_laid_out_once_reach_their_entry_point(b):
    L = b.lib()
    at = ctypes.addressof
    w, c = b._Weight(P, P, None, None, 8, 64, 0, 0, 0, None), _cache(b)
    q = b._KV8Queries(P, P, P, P, 0.125, 0, 2, 4, 256, 2, 4, 1, 64, 0)

    def run(entry, pointers, ints=(), n=0):
        call = b._Call((ctypes.c_void_p * 10)(*pointers), n, (ctypes.c_int * 6)(*ints), 0.0, entry)
        return L.w4a4_run_call(ctypes.byref(call), None)

    names = b._Prepared.ENTRIES
    assert names.index("w4a4_linear_w4a16") == 6 and names.index("w4a4_kv8_attention") == 10
    assert run(6, (P, at(w), None, P), (0, 0, 64, 64, 0)) == 0 and run(6, (P, at(w), None, P), (0, 4, 64, 32, 0)) == -1 and run(6, (P, at(w), P + 2, P), (0, 4, 64, 64, 0)) == -2
    assert run(6, (P, at(w), None, P), (2, 4, 64, 64, 0)) == -1 and run(6, (P, at(w), None, P), (0, 4, 64, 64, 9)) == -1
    plan = [P, P, P, P, P, 2 * P, 2 * P, P, P, P]
    assert run(7, plan, (4, 8, 16, 24, 4)) == -2 and run(7, plan, (4, 8, 0, 16, 4)) == -1 and run(7, plan, (4, -1, 16, 16, 4)) == -1 and run(7, plan, (4, 8, 16, 16, -1)) == -1
    assert run(8, (at(c), P, P, P), (0, 0, 128, 128)) == 0 and run(8, (at(c), P, P, P), (0, 4, 64, 128)) == -1 and run(8, (at(c), P, P, P), (0, 4, 128, 132)) == -2
    assert run(9, (at(c), P, P, P), (0, 0)) == 0 and run(9, (at(c), P, P, P), (4, 2)) == -1 and run(9, (at(c), P, P + 4, P), (4, 0)) == -2
    assert run(10, (at(c), at(q), None, None, None)) == -1 and run(10, (at(c), at(q), P + 2, None, None)) == -2
    q.width, q.context = 10000, 150000
    assert run(10, (at(c), at(q), P, None, P), n=16) == -3
    q.tokens = 0
    assert run(10, (at(c), at(q), None, None, None)) == 0
