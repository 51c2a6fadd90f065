"""The entry points around 4-bit weights and caches refuse bad arguments on the host, before anything is enqueued, with the documented status."""
import ctypes as C
import math
import os
import random

import pytest

P = C.c_void_p
OK, NULL, SHAPE, ALIGN, PARAM, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 6, 7
FP4 = -4


@pytest.fixture(scope="module")
def lib():
    from paper_2510_00206_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    assert binding.KV_FP4 == FP4
    return binding.load_library()


def _changed(good, **kw):
    return list({**good, **kw}.values())


def _cache(**kw):
    from paper_2510_00206_amd import binding
    good = dict(k=0x1000, v=0x1000, k_exp=0x1000, v_exp=0x1000, pages=8, page=16, heads=2, dim=64, fp8=FP4)
    return C.byref(binding.CacheArrays(*_changed(good, **kw)))


@pytest.mark.parametrize("name", ["lora_weights_write", "lora_weights_read"])
def test_weights(lib, name):
    p = P(0x1000)
    keys = ("W", "N", "K", "codes", "exps") if name.endswith("write") else ("codes", "exps", "N", "K", "W")
    good = {**{k: 64 if k in "NK" else p for k in keys}, "stream": None}
    f = lambda **kw: getattr(lib, name)(*_changed(good, **kw))
    for k in ("W", "codes", "exps"):
        assert f(**{k: None}) == NULL, k
        assert f(**{k: P(0x1008)}) == ALIGN, k
    assert [f(N=0), f(K=0), f(N=-64), f(K=1 << 31), f(N=1 << 40)] == [SHAPE] * 5
    assert [f(N=96), f(K=32), f(K=100), f(N=1 << 23), f(K=1 << 23)] == [UNSUPPORTED] * 5


def test_layer(lib):
    p = P(0x1000)
    good = dict(X=p, codes=p, exps=p, A=p, B=p, ids=p, ranks=None, s=p, M=8, K=64, N=128, r=16, P=3, Y=p, S=p, stream=None)
    f = lambda **kw: lib.lora_requests_quantised_fwd(*_changed(good, **kw))
    assert f(M=0) == OK and f(M=0, X=None, ids=None, Y=None, S=None) == OK
    none = dict(A=None, B=None, ids=None, s=None, S=None, P=0, r=0)
    assert f(M=0, **none) == OK and f(**{**none, "X": None}) == NULL and f(**{**none, "Y": None}) == NULL and f(**{**none, "codes": None}) == NULL
    for name in ("X", "codes", "exps", "A", "B", "ids", "s", "Y", "S"):
        assert f(**{name: None}) == NULL, name
    assert [f(M=-1), f(K=0), f(N=-64), f(P=-1), f(M=1 << 31), f(P=1 << 31)] == [SHAPE] * 6
    assert [f(K=96), f(N=100), f(r=8), f(r=48), f(K=1 << 23), f(N=1 << 23), f(M=1 << 21)] == [UNSUPPORTED] * 7
    for name in ("X", "codes", "exps", "A", "B", "Y", "S"):
        assert f(**{name: P(0x1008)}) == ALIGN, name
    assert f(ids=P(0x1002)) == ALIGN and f(ranks=P(0x1001)) == ALIGN and f(s=P(0x1002)) == ALIGN


@pytest.mark.parametrize("fp8", [0, 1, FP4])
def test_append(lib, fp8):
    p, c = P(0x1000), _cache(fp8=fp8)
    good = dict(cache=c, q=p, k=p, v=p, gq=p, gk=p, cos=p, sin=p, pos=p, slots=p, M=4, H=4, rot=64, positions=10, ldq=256, ldk=128, ldv=128, ldqo=256, eps=1e-6,
                inter=0, qo=p, stream=None)
    f = lambda **kw: lib.lora_kv_cache_append(*_changed(good, **kw))
    assert f(M=0) == OK and f(M=0, q=None, k=None, v=None, pos=None, slots=None, qo=None, gq=None, gk=None) == OK
    assert f(M=0, positions=0, cos=None, sin=None) == OK
    for name in ("cache", "q", "k", "v", "gq", "gk", "cos", "sin", "pos", "slots", "qo"):
        assert f(**{name: None}) == NULL, name
    assert [f(M=-1), f(H=0), f(positions=-1), f(positions=1 << 31), f(ldq=248), f(ldk=120), f(ldv=132), f(ldqo=260)] == [SHAPE] * 8
    assert [f(rot=8), f(rot=80), f(rot=40), f(H=1025), f(M=1 << 26)] == [UNSUPPORTED] * 5
    assert [f(eps=0.0), f(eps=-1.0), f(eps=float("nan")), f(eps=float("inf"))] == [PARAM] * 4
    for name in ("q", "k", "v", "gq", "gk", "cos", "sin", "qo"):
        assert f(**{name: P(0x1008)}) == ALIGN, name
    assert f(pos=P(0x1002)) == ALIGN and f(slots=P(0x1004)) == ALIGN
    if fp8:
        assert f(cache=_cache(fp8=fp8, k_exp=None)) == NULL and f(cache=_cache(fp8=fp8, v_exp=None)) == NULL
    for bad in (dict(page=8), dict(page=48), dict(dim=72), dict(heads=1025)):
        assert f(cache=_cache(fp8=fp8, **bad)) == UNSUPPORTED, bad


def test_cache_in_4_bits(lib):
    """Entries in 32s; everything else as for the other forms.  Any other number but 0 still is fp8."""
    p = P(0x1000)
    w = lambda c, M=4: lib.lora_kv_cache_write(c, p, p, 512, 512, p, M, None)
    r = lambda c, M=4: lib.lora_kv_cache_read(c, p, M, p, p, 512, 512, None)
    a = lambda c, T=4: lib.lora_paged_attn_fwd(p, c, p, p, p, T, 8, 2, 5, 1024, 5, 1024, 2, 80, 0.1, 0, p, p, 1 << 30, None)
    for f in (w, r):
        assert f(_cache(), 0) == OK and f(_cache(dim=96), 0) == OK and f(_cache(dim=80, fp8=1), 0) == OK and f(_cache(dim=80, fp8=4), 0) == OK
        assert f(_cache(dim=80), 0) == UNSUPPORTED and f(_cache(dim=16), 0) == UNSUPPORTED and f(_cache(k_exp=None)) == NULL and f(_cache(v_exp=None)) == NULL
        assert f(_cache(k=0x1008)) == ALIGN and f(_cache(k_exp=0x1004)) == ALIGN and f(_cache(v_exp=0x1008)) == ALIGN
    assert a(_cache(), 0) == OK and a(_cache(dim=96)) == UNSUPPORTED and a(_cache(dim=80)) == UNSUPPORTED and a(_cache(v_exp=None)) == NULL
    for dim in (64, 128):
        one, other = (lib.lora_paged_attn_workspace_bytes(_cache(dim=dim, heads=8, fp8=form), 4, 32, 4, 1, 131072, 0) for form in (1, FP4))
        assert one == other > 256


def test_workspace_of_smaller_steps(lib):
    """What the query returns for a step is enough for every smaller one, which may be cut into more parts."""
    rng = random.Random(3)
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.9))))
    for _ in range(4000):
        G, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 8, 33, 40))
        cache = _cache(heads=G, dim=rng.choice((64, 128)))
        B, new, kv, window = log(1, 200), rng.choice((1, log(1, 600))), log(1, 200000), rng.choice((0, 0, log(1, 5000)))
        T = log(1, B * new)
        B2, new2, kv2 = log(1, B), log(1, new), log(1, kv)
        T2 = log(1, min(T, B2 * new2))
        big, small = (lib.lora_paged_attn_workspace_bytes(cache, t, G * group, b, n, k, window) for t, b, n, k in ((T, B, new, kv), (T2, B2, new2, kv2)))
        assert 256 <= small <= big, (G, group, (T, B, new, kv), (T2, B2, new2, kv2), window)


def test_in_place_with_another_stride(lib):
    """Rows written over rows that are still read are refused: queries (and keys) in place keep their stride."""
    p, other = P(0x1000), P(0x800000)
    base = dict(gq=p, gk=p, cos=p, sin=p, pos=p)
    append = dict(cache=_cache(), q=p, k=other, v=other, **base, slots=p, M=4, H=4, rot=64, positions=10, ldq=512, ldk=128, ldv=128, ldqo=256, eps=1e-6, inter=0, qo=p,
                  stream=None)
    f = lambda **kw: lib.lora_kv_cache_append(*_changed(append, **kw))
    assert f() == SHAPE and f(ldq=256, ldqo=512) == SHAPE and f(M=0) == OK and f(M=0, ldqo=512) == OK
    rope = dict(q=p, k=other, **base, M=4, H=4, G=2, D=64, rot=64, positions=10, ldq=512, ldk=128, ldqo=512, ldko=128, eps=1e-6, inter=0, qo=p, ko=other, stream=None)
    f = lambda **kw: lib.lora_qk_norm_rope_fwd(*_changed(rope, **kw))
    assert f(ldqo=256) == SHAPE and f(ldko=256) == SHAPE and f(ldqo=256, M=0) == OK


def test_layer_tiles(lib):
    """The kinds of tile that the layer's tests are meant for are those that these sizes take, and every kind is among them."""
    from paper_2510_00206_amd import binding
    from quant_util import WRAPPED
    seen = set()
    for tile, M, K, N in WRAPPED:
        t = binding.lora_debug_quantised_tiles(M, K, N, 32, 5)
        assert (t.rows, t.columns) == tile and K // 128 > 2 * t.ring_blocks and not t.own_term, (tile, M, K, N, t.rows, t.columns, t.ring_blocks)
        seen.add((tile, t.ring_blocks, K % 128))
    for M in list(range(1, 70)) + [80, 100, 130, 200, 260, 300, 520, 700, 1300, 2050]:
        for K in (64, 256, 1024, 4096, 4160, 14336):
            for N in (64, 1024, 4096, 4160, 6144, 14336):
                t = binding.lora_debug_quantised_tiles(M, K, N)
                assert all(((t.rows, t.columns), t.ring_blocks, half) in seen for half in (0, 64)), (M, K, N)
    one = [binding.lora_debug_quantised_tiles(1, 1024, 1024, r, P).own_term for r, P in ((16, 4), (32, 4), (64, 4), (16, 0))]
    assert one == [1, 1, 0, 0]
    f = lib.lora_debug_quantised_tiles
    out = binding.QuantisedTiles()
    assert f(8, 64, 64, 16, 1, None) == NULL and f(-1, 64, 64, 16, 1, C.byref(out)) == SHAPE and f(8, 32, 64, 16, 1, C.byref(out)) == UNSUPPORTED
    assert f(0, 64, 64, 16, 1, C.byref(out)) == OK and out.rows == out.columns == out.ring_blocks == 0
