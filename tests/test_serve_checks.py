"""The entry points around served adapters refuse bad arguments on the host, before anything is enqueued, with the documented status."""
import ctypes as C
import os
import random

import pytest

P = C.c_void_p
OK, NULL, SHAPE, ALIGN, PARAM, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 6, 7


@pytest.fixture(scope="module")
def lib():
    from paper_2510_00206_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load_library()


def _changed(good, **kw):
    return list({**good, **kw}.values())


def test_requests(lib):
    p = P(0x1000)
    good = dict(X=p, W=p, A=p, B=p, ids=p, ranks=None, s=p, M=8, K=64, N=128, r=16, P=3, Y=p, S=p, stream=None)
    f = lambda **kw: lib.lora_requests_fwd(*_changed(good, **kw))
    assert f(M=0) == OK and f(M=0, X=None, ids=None, Y=None, S=None) == OK
    for name in ("X", "W", "A", "B", "ids", "s", "Y", "S"):
        assert f(**{name: None}) == NULL, name
    assert [f(M=-1), f(K=0), f(N=-64), f(P=0), f(M=1 << 31)] == [SHAPE] * 5
    assert [f(K=96), f(N=100), f(r=8), f(r=48), f(K=1 << 23), f(M=1 << 21)] == [UNSUPPORTED] * 6
    for name in ("X", "W", "A", "B", "Y", "S"):
        assert f(**{name: P(0x1008)}) == ALIGN, name
    assert f(ids=P(0x1002)) == ALIGN and f(ranks=P(0x1001)) == ALIGN and f(s=P(0x1002)) == ALIGN


ROPE = dict(q=P(0x1000), k=P(0x1000), gq=P(0x1000), gk=P(0x1000), cos=P(0x1000), sin=P(0x1000), pos=P(0x1000))
SIZES = dict(M=4, H=4, G=2, D=64, rot=64, positions=10)


def test_norm_rope(lib):
    p = P(0x1000)
    good = {**ROPE, **SIZES, **dict(ldq=256, ldk=128, ldqo=256, ldko=128, eps=1e-6, inter=0, qo=p, ko=p, stream=None)}
    f = lambda **kw: lib.lora_qk_norm_rope_fwd(*_changed(good, **kw))
    assert f(M=0, q=None, k=None, pos=None, qo=None, ko=None) == OK
    for name in ("q", "k", "gq", "gk", "cos", "sin", "pos", "qo", "ko"):
        assert f(**{name: None}) == NULL, name
    assert [f(M=-1), f(H=0), f(G=0), f(D=0), f(positions=-1), f(ldq=248), f(ldk=120), f(ldqo=260), f(ldko=132)] == [SHAPE] * 9
    assert [f(D=72, rot=32, ldq=1024, ldk=1024), f(D=272, ldq=4096, ldk=4096), f(rot=8), f(rot=80), f(rot=40), f(H=1025), f(M=1 << 26)] == [UNSUPPORTED] * 7
    assert [f(eps=0.0), f(eps=-1.0), f(eps=float("nan")), f(eps=float("inf"))] == [PARAM] * 4
    for name in ("q", "k", "gq", "gk", "cos", "sin", "qo", "ko"):
        assert f(**{name: P(0x1008)}) == ALIGN, name
    assert f(pos=P(0x1002)) == ALIGN


def test_norm_rope_backward(lib):
    p, need = P(0x1000), lib.lora_qk_norm_rope_workspace_bytes(4, 4, 2, 64)
    assert need >= 256 and lib.lora_qk_norm_rope_workspace_bytes(4, 4, 2, 72) == 0 and lib.lora_qk_norm_rope_workspace_bytes(-1, 4, 2, 64) == 0
    good = {**ROPE, **dict(dqo=p, dko=p), **SIZES, **dict(ldq=256, ldk=128, lddqo=256, lddko=128, lddq=256, lddk=128, eps=1e-6, inter=0, dq=p, dk=p,
                                                         dgq=p, dgk=p, acc=0, ws=p, n=need, stream=None)}
    f = lambda **kw: lib.lora_qk_norm_rope_bwd(*_changed(good, **kw))
    for name in ("q", "k", "gq", "gk", "cos", "sin", "pos", "dqo", "dko", "dq", "dk", "dgq", "dgk", "ws"):
        assert f(**{name: None}) == NULL, name
    assert [f(lddqo=248), f(lddko=120), f(lddq=255), f(lddk=64), f(M=-1)] == [SHAPE] * 5
    assert f(n=need - 1) == WORKSPACE and f(eps=0.0) == PARAM and f(ws=P(0x1080)) == ALIGN and f(dgq=P(0x1004)) == ALIGN
    # the planes of partial sums: never more than the query provides for
    for M in (1, 5, 300, 4096, 100000):
        assert lib.lora_qk_norm_rope_workspace_bytes(M, 64, 8, 128) <= 1024 * 2 * 128 * 4


def _cache(**kw):
    from paper_2510_00206_amd import binding
    good = dict(k=0x1000, v=0x1000, k_exp=0x1000, v_exp=0x1000, pages=8, page=16, heads=2, dim=64, fp8=1)
    return C.byref(binding.CacheArrays(*_changed(good, **kw)))


def test_cache(lib):
    p = P(0x1000)
    w = lambda c, k=p, v=p, ldk=128, ldv=128, slots=p, M=4: lib.lora_kv_cache_write(c, k, v, ldk, ldv, slots, M, None)
    r = lambda c, k=p, v=p, ldk=128, ldv=128, slots=p, M=4: lib.lora_kv_cache_read(c, slots, M, k, v, ldk, ldv, None)
    for f in (w, r):
        assert f(_cache(), M=0, k=None, v=None, slots=None) == OK
        for bad in (dict(k=None), dict(v=None), dict(k_exp=None), dict(v_exp=None)):
            assert f(_cache(**bad)) == NULL
        assert f(_cache(), k=None) == NULL and f(_cache(), v=None) == NULL and f(_cache(), slots=None) == NULL and f(None) == NULL
        for bad in (dict(pages=0), dict(page=0), dict(heads=0), dict(dim=-16)):
            assert f(_cache(**bad)) == SHAPE
        for bad in (dict(page=8), dict(page=48), dict(page=2048), dict(dim=72), dict(dim=272), dict(heads=1025), dict(pages=1 << 31)):
            assert f(_cache(**bad)) == UNSUPPORTED, bad
        assert [f(_cache(), ldk=120), f(_cache(), ldv=132), f(_cache(), M=-1)] == [SHAPE] * 3
        assert [f(_cache(k=0x1008)), f(_cache(v=0x1004)), f(_cache(), k=P(0x1002)), f(_cache(), slots=P(0x1004))] == [ALIGN] * 4
        assert f(_cache(), M=1 << 27) == UNSUPPORTED


def test_attention(lib):
    p = P(0x1000)
    good = dict(q=p, cache=_cache(), table=p, offsets=p, kv_lens=p, T=4, H=8, B=2, max_pages=5, ldq=512, ldt=5, ldo=512, max_new=2, max_kv=80, scale=0.1,
                window=0, out=p, ws=p, n=1 << 30, stream=None)
    f = lambda **kw: lib.lora_paged_attn_fwd(*_changed(good, **kw))
    assert f(T=0, q=None, out=None) == OK and f(B=0) == OK and f(max_new=0) == OK
    for name in ("q", "table", "offsets", "kv_lens", "out", "ws"):
        assert f(**{name: None}) == NULL, name
    assert [f(T=-1), f(B=-1), f(H=0), f(H=7), f(max_new=-1), f(max_kv=-1), f(window=-1), f(max_pages=-1), f(ldt=4), f(ldq=504), f(ldo=516)] == [SHAPE] * 11
    assert [f(cache=_cache(dim=128), ldq=1024, ldo=1024, T=0), f(cache=_cache(dim=96))] == [OK, UNSUPPORTED]
    assert [f(T=1 << 30), f(max_kv=1 << 30), f(window=1 << 30), f(max_pages=1 << 27, ldt=1 << 27)] == [UNSUPPORTED] * 4
    assert [f(scale=0.0), f(scale=-1.0), f(scale=float("nan")), f(scale=float("inf"))] == [PARAM] * 4
    assert [f(q=P(0x1008)), f(out=P(0x1008)), f(ws=P(0x1010)), f(table=P(0x1002)), f(offsets=P(0x1001)), f(kv_lens=P(0x1002))] == [ALIGN] * 6


def test_attention_workspace(lib):
    """A long range of few rows is cut into parts, whose results the workspace holds; a smaller one is refused."""
    p, c = P(0x1000), _cache(dim=128, heads=8)
    need = lambda T, H, B, new, kv, window=0: lib.lora_paged_attn_workspace_bytes(c, T, H, B, new, kv, window)
    assert need(1, 32, 1, 1, 100) >= 256 and need(1, 32, 1, 1, 131072) > 32 * 129 * 4 and need(-1, 32, 1, 1, 100) == 0 and need(1, 30, 1, 1, 100) == 0
    assert need(1, 32, 1, 1, 131072, 500) < need(1, 32, 1, 1, 131072)
    n = need(1, 32, 1, 1, 131072)
    call = lambda size: lib.lora_paged_attn_fwd(p, c, p, p, p, 1, 32, 1, 10000, 4096, 10000, 4096, 1, 131072, 0.1, 0, p, p, size, None)
    assert call(n - 1) == WORKSPACE


def test_attention_workspace_serves_smaller_steps(lib):
    """What the query returns never falls as a step grows: one workspace, for the largest, is enough for all."""
    rng = random.Random(5)
    size = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))
    for _ in range(3000):
        heads, dim = rng.choice((1, 2, 8, 16)), rng.choice((64, 128))
        c, H, window = _cache(dim=dim, heads=heads), heads * rng.choice((1, 4, 7, 16, 40)), rng.choice((0, 0, size(1, 20000)))
        B, new, kv = size(1, 200), size(1, 2000), size(1, 150000)
        T = size(1, B * new)
        B1, new1, kv1 = size(1, B), size(1, new), size(1, kv)
        T1 = size(1, min(T, B1 * new1))
        large, small = (lib.lora_paged_attn_workspace_bytes(c, t, H, b, n, k, window) for t, b, n, k in ((T, B, new, kv), (T1, B1, new1, kv1)))
        assert 256 <= small <= large, (heads, dim, H, window, (T, B, new, kv), (T1, B1, new1, kv1))


def test_cache_rows_of_a_launch(lib):
    """Rows whose workgroups of 256 threads, 32 to a head, would pass the 2^32 threads of a launch are refused."""
    p = P(0x1000)
    for heads in (1, 3, 7, 8, 1000):
        first = next(M for M in range((1 << 27) // heads - 20, (1 << 27) // heads + 20) if (M * heads * 32 + 255) // 256 * 256 >= 1 << 32)
        c = _cache(dim=256, heads=heads)
        assert lib.lora_kv_cache_write(c, p, p, 256 * heads, 256 * heads, p, first, None) == UNSUPPORTED, heads
        assert lib.lora_kv_cache_read(c, p, first, p, p, 256 * heads, 256 * heads, None) == UNSUPPORTED, heads


def test_attention_sizes_that_wrap(lib):
    """Sizes whose products pass 64 bits are refused as other large ones are."""
    p, c = P(0x1000), _cache()
    good = dict(q=p, cache=c, table=p, offsets=p, kv_lens=p, T=4, H=8, B=2, max_pages=5, ldq=512, ldt=5, ldo=512, max_new=2, max_kv=80, scale=0.1, window=0, out=p,
                ws=p, n=1 << 30, stream=None)
    for bad in (dict(T=1 << 61), dict(T=(1 << 61) + 4), dict(max_new=1 << 61), dict(max_new=(1 << 61) + 2), dict(max_pages=1 << 60, ldt=1 << 60),
                dict(max_pages=(1 << 60) + 5, ldt=1 << 62)):
        assert lib.lora_paged_attn_fwd(*_changed(good, **bad)) == UNSUPPORTED, bad
    assert lib.lora_paged_attn_workspace_bytes(c, 1 << 61, 8, 2, 2, 80, 0) == 0
    assert lib.lora_paged_attn_workspace_bytes(c, 4, 8, 2, 1 << 61, 80, 0) == 0
