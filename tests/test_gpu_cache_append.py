"""Norm, rotation and the writing of the cache in one call: queries within their bound, codes and exponents bit for bit those of the 64-bit form, rows and
slots outside left out, in every form of the cache."""
import pytest
import torch

from paper_2510_00206_amd import binding
from quant_util import quantised4, widened4
from serve_util import BF16, F32, F64, U16, U32, gen, norm_rope, normal, quantised, turn, widened, within

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -20


def _setup(M, H, G, D, rot, page, form, norm, seed, positions=50, spread=True):
    g = gen(seed)
    qkv = normal(g, (M, (H + 2 * G) * D + 16))
    q, k, v = (qkv[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    if spread:
        v.copy_((v.float() * torch.exp2(torch.randint(-20, 20, (M, G, 1), generator=g).float())).to(BF16))
    gq, gk = (normal(g, (D,), 0.3, 1.0) for _ in range(2)) if norm else (None, None)
    ang = torch.rand((positions, rot // 2), generator=g, dtype=F64) * 6.3
    cos, sin = ang.cos().to(F32), ang.sin().to(F32)
    pos = torch.randint(0, positions, (M,), generator=g, dtype=torch.int32)
    pages = M // page + 2
    slots = torch.randperm(pages * page, generator=g)[:M]
    cache = binding.KVCache.empty(pages, page, G, D, fp8=form == "fp8", fp4=form == "fp4")
    for t in cache.tensors:
        if t is not None:
            t.view(torch.uint8).fill_(0x11)
    return qkv, q, k, v, gq, gk, cos, sin, pos, slots, cache


def _ref(x, gamma, cos, sin, pos, inter):
    """In 64 bits, and its bound in fp32 with one rounding."""
    if gamma is not None:
        return norm_rope(x.to(F64), gamma.to(F64), cos, sin, pos, EPS, inter)
    known = ((pos >= 0) & (pos < cos.shape[0]))[:, None, None]
    at = pos.clamp(0, cos.shape[0] - 1).long()
    c, s = (t.to(F64)[at][:, None] for t in (cos, sin))
    y = torch.where(known, turn(x.to(F64), c, s, inter), torch.zeros(x.shape, dtype=F64))
    return y, U16 * y.abs() + 4 * U32 * 2 * x.to(F64).abs().amax(-1, keepdim=True)


def _held(cache, slots):
    p, o = (slots // cache.page).cuda(), (slots % cache.page).cuda()
    return [None if t is None else t[p, :, o].cpu() for t in cache.tensors]


def _compare(form, cache, slots, k, k_bound, v, label):
    hk, hv, ke, ve = _held(cache, slots)
    if form == "bf16":
        within(hk, k, k_bound, (label, "keys"))
        assert torch.equal(hv, v.to(BF16))
        return
    for x, codes, exps in ((k, hk, ke), (v.to(F64), hv, ve)):
        if form == "fp4":
            rc, re = quantised4(x)
            assert torch.equal(exps, re), (label, "exponents")
            assert torch.equal(codes, rc), (label, "codes", int((codes != rc).sum()))
        else:
            top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
            e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0)), torch.zeros_like(top)).clamp(min=-117)
            assert torch.equal(exps.to(F64), e + 127), (label, "exponents")
            a = x / torch.exp2(e)[..., None]
            step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
            assert torch.equal(codes.view(torch.float8_e4m3fn).to(F64), torch.round(a / step) * step), (label, "codes")


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("M,H,G,D,rot,page,form,inter", [
    (1, 1, 1, 64, 64, 16, "fp4", False), (1, 32, 8, 128, 128, 16, "fp4", False), (5, 6, 3, 32, 16, 32, "fp4", True), (37, 4, 2, 96, 48, 16, "fp4", False),
    (100, 32, 8, 128, 128, 16, "fp4", False), (33, 2, 1, 256, 256, 128, "fp4", True), (300, 8, 8, 64, 32, 64, "fp4", False),
    (1, 8, 2, 128, 128, 16, "fp8", False), (61, 7, 7, 80, 80, 16, "fp8", True), (130, 16, 4, 128, 64, 32, "fp8", False), (20, 4, 4, 16, 16, 16, "fp8", False),
    (1, 4, 1, 16, 16, 16, "bf16", False), (77, 12, 3, 208, 112, 64, "bf16", True), (260, 32, 8, 128, 128, 16, "bf16", False), (9, 1, 5, 64, 64, 1024, "bf16", False)])
def test_against_64_bits(M, H, G, D, rot, page, form, inter, norm):
    print("append", M, H, G, D, rot, page, form, inter, norm, flush=True)
    qkv, q, k, v, gq, gk, cos, sin, pos, slots, cache = _setup(M, H, G, D, rot, page, form, norm, M + D)
    dev = qkv.cuda()
    dq, dk, dv = (dev[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    before = [None if t is None else t.clone() for t in cache.tensors]
    out = torch.full((M, H, D), 7.0, dtype=BF16, device="cuda")
    args = [t if t is None else t.cuda() for t in (cos, sin, pos, slots)]
    binding.lora_kv_cache_append(cache, dq, dk, dv, *args, gq=None if gq is None else gq.cuda(), gk=None if gk is None else gk.cuda(), eps=EPS, interleaved=inter,
                                 q_out=out)
    torch.cuda.synchronize()
    ref, bound = _ref(q, gq, cos, sin, pos, inter)
    within(out, ref, bound, "queries")
    kref, kbound = _ref(k, gk, cos, sin, pos, inter)
    _compare(form, cache, slots, kref, kbound, v, (M, H, G, D, form))
    # the other slots as they were
    left = torch.ones((cache.pages, cache.page), dtype=torch.bool)
    left[slots // page, slots % page] = False
    for t, b in zip(cache.tensors, before):
        if t is not None:
            assert torch.equal(t.view(torch.uint8).transpose(1, 2)[left.cuda()], b.view(torch.uint8).transpose(1, 2)[left.cuda()])
    # queries in place
    binding.lora_kv_cache_append(cache, dq, dk, dv, *args, gq=None if gq is None else gq.cuda(), gk=None if gk is None else gk.cuda(), eps=EPS, interleaved=inter,
                                 q_out=dq)
    assert torch.equal(dq, out)


@pytest.mark.parametrize("form", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("M", [3, 70])
def test_rows_and_slots_outside(form, M):
    """A position outside the tables: zeros for query and keys (values are held); a slot outside the cache: nothing is held, the query comes out.  Rows outside both may
    hold anything."""
    H, G, D = 4, 2, 64
    qkv, q, k, v, gq, gk, cos, sin, pos, slots, cache = _setup(M, H, G, D, 64, 16, form, True, 9)
    pos[0], pos[1] = -1, 50
    good = slots.clone()
    slots[1], slots[2] = -1, cache.pages * 16
    q[1], k[1], v[1] = float("nan"), float("inf"), float("nan")
    before = [None if t is None else t.clone() for t in cache.tensors]
    out = binding.lora_kv_cache_append(cache, q.cuda().contiguous(), k.cuda().contiguous(), v.cuda().contiguous(), cos.cuda(), sin.cuda(), pos.cuda(), slots.cuda(),
                                       gq=gq.cuda(), gk=gk.cuda(), eps=EPS)
    assert int((out[:2] != 0).sum()) == 0 and bool(torch.isfinite(out).all())
    keep = [0] + list(range(3, M))
    kref, kbound = _ref(k, gk, cos, sin, pos, False)
    _compare(form, cache, slots[keep], kref[keep], kbound[keep], v[keep], (form, M))
    for t, b in zip(cache.tensors, before):
        if t is not None:
            p, o = (good[1:3] // 16).cuda(), (good[1:3] % 16).cuda()
            assert torch.equal(t.view(torch.uint8)[p, :, o], b.view(torch.uint8)[p, :, o])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_borders_without_rotation(D):
    """At position 0, without a norm, what goes in is what is held: halfway between two codes, and right past the range of a power of two."""
    M, G = 40, 2
    g = gen(D)
    steps = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.5, 1.0, 2.0, 3.0, 4.0, 0.0, 5.96875, 3.015625, 0.251953125, 2.515625])
    k = steps[torch.randint(0, len(steps), (M, G, D), generator=g)] * (1 - 2 * torch.randint(0, 2, (M, G, D), generator=g)) * \
        torch.exp2(torch.randint(-100, 100, (M, G, 1), generator=g).float())
    k = k.to(BF16)
    k[0, 0, :32] = 0
    k[1, 1, 3], k[2, 0, D - 1] = float("inf"), float("nan")
    cos, sin = torch.ones((1, D // 2), device="cuda"), torch.zeros((1, D // 2), device="cuda")
    cache = binding.KVCache.empty(4, 16, G, D, fp4=True)
    slots, pos = torch.arange(M), torch.zeros(M, dtype=torch.int32, device="cuda")
    binding.lora_kv_cache_append(cache, k.cuda(), k.cuda(), k.cuda(), cos, sin, pos, slots.cuda())
    hk, hv, ke, ve = _held(cache, slots)
    rc, re = quantised4(k)
    sure = torch.ones(M, dtype=torch.bool)
    sure[1:3] = False                                                   # (0 x infinity of a pair's other entry)
    assert torch.equal(hv, rc) and torch.equal(ve, re)
    # (a zero of either sign may come out of a product with the sine)
    assert torch.equal(ke[sure], re[sure]) and torch.equal(widened4(hk, ke)[sure], widened4(rc, re)[sure])
    for i, (row, head, entry) in enumerate(((1, 1, 3), (2, 0, D - 1))):
        other = (entry + D // 2) % D
        assert int(ke[row, head, entry // 32]) == 255 and int(ke[row, head, other // 32]) == 255


@pytest.mark.parametrize("M,G,D,page", [(1, 1, 32, 16), (5, 3, 64, 32), (100, 8, 128, 16), (33, 1, 256, 128), (64, 4, 224, 16), (50, 5, 96, 1024)])
def test_write_and_read_in_4_bits(M, G, D, page):
    print("cache in 4 bits", M, G, D, page, flush=True)
    g = gen(M + D)
    pages = M // page + 2
    spread = torch.exp2(torch.randint(-60, 60, (M, G, 1), generator=g).float())
    kv = torch.stack((normal(g, (M, G, D)).float() * spread, normal(g, (M, G, D)).float() / spread), 1).to(BF16)
    kv[0, 0, 0] = 0
    kv[0, 1, 0, :2] = torch.tensor([float("inf"), -float("inf")])
    kv[M - 1, 0, G - 1, D - 1] = float("nan")
    slots = torch.randperm(pages * page, generator=g)[:M]
    cache = binding.KVCache.empty(pages, page, G, D, fp4=True)
    for t in cache.tensors:
        t.fill_(0x11)
    dev = kv.cuda()
    outside = slots.clone()
    if M > 4:
        outside[2], outside[3] = -7, pages * page
    binding.lora_kv_cache_write(cache, dev[:, 0], dev[:, 1], outside.cuda())
    p, o = slots // page, slots % page
    back = binding.lora_kv_cache_read(cache, outside.cuda())
    for i in range(2):
        codes, exps = cache.tensors[i].cpu(), cache.tensors[2 + i].cpu()
        rc, re = quantised4(kv[:, i])
        if M > 4:
            rc[2:4], re[2:4] = 0x11, 0x11
        assert torch.equal(exps[p, :, o], re) and torch.equal(codes[p, :, o], rc)
        left = torch.ones((pages, page), dtype=torch.bool)
        left[p, o] = False
        assert bool((codes.transpose(1, 2)[left] == 0x11).all()) and bool((exps.transpose(1, 2)[left] == 0x11).all())
        ref = widened4(rc, re)
        if M > 4:
            ref[2:4] = 0
        got, nan = back[i].cpu().to(F64), torch.isnan(ref)
        assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], ref[~nan])


@pytest.mark.parametrize("form", ["bf16", "fp4"])
def test_a_launch_and_another(form):
    """More rows than a launch has (2^24 of one query head and one of keys and values): the first ones, those on either side of 2^24 and the last ones; the others of zeros."""
    M, D, page = (1 << 24) + 37, 32, 1024
    g = gen(12)
    rows = torch.cat([torch.arange(20), torch.arange((1 << 24) - 20, M)])
    qkv = torch.zeros((M, 3 * D), dtype=BF16, device="cuda")
    some = normal(g, (rows.numel(), 3 * D))
    qkv[rows.cuda()] = some.cuda()
    pos = torch.zeros((M,), dtype=torch.int32, device="cuda")
    slots = torch.arange(M, device="cuda").flip(0)
    ang = torch.rand((1, D // 2), generator=g, dtype=F64) * 6.3
    cos, sin = ang.cos().to(F32), ang.sin().to(F32)
    gq, gk = (normal(g, (D,), 0.3, 1.0) for _ in range(2))
    cache = binding.KVCache.empty(M // page + 1, page, 1, D, fp4=form == "fp4")
    q, k, v = (qkv[:, i * D:(i + 1) * D].unflatten(1, (1, D)) for i in range(3))
    out = binding.lora_kv_cache_append(cache, q, k, v, cos.cuda(), sin.cuda(), pos, slots, gq=gq.cuda(), gk=gk.cuda(), eps=EPS)
    sq, sk, sv = (some[:, i * D:(i + 1) * D].unflatten(1, (1, D)) for i in range(3))
    at = torch.zeros(rows.numel(), dtype=torch.int32)
    ref, bound = _ref(sq, gq, cos, sin, at, False)
    within(out[rows.cuda()], ref, bound, "queries")
    kref, kbound = _ref(sk, gk, cos, sin, at, False)
    _compare(form, cache, slots[rows.cuda()].cpu(), kref, kbound, sv, form)
    assert int((out[20:(1 << 24) - 20] != 0).sum()) == 0            # (zeros of either sign: 0 x a negative cosine)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("form", ["bf16", "fp8", "fp4"])
def test_entries_past_the_rotation_stand_alone(form, inter, norm):
    """Entries that are not turned have no pair: infinity and NaN there leave the others as they are, and without a norm come out as they went in."""
    M, H, G, D, rot = 5, 3, 2, 64, 32
    qkv, q, k, v, gq, gk, cos, sin, pos, slots, cache = _setup(M, H, G, D, rot, 16, form, norm, 77)
    for x in (q, k):
        x[0, 1, 41], x[1, 0, 40], x[1, 0, 55], x[2, 1, 63] = float("inf"), -float("inf"), float("inf"), float("nan")
        x[3, 0, 36], x[3, 0, 37] = 0.0, -0.0
    dq, dk, dv = (t.cuda().contiguous() for t in (q, k, v))
    out = binding.lora_kv_cache_append(cache, dq, dk, dv, cos.cuda(), sin.cuda(), pos.cuda(), slots.cuda(), gq=None if gq is None else gq.cuda(),
                                       gk=None if gk is None else gk.cuda(), eps=EPS, interleaved=inter).cpu()

    def close(got, x, gamma):
        ref, _ = _ref(x, gamma, cos, sin, pos, inter)
        top = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).to(F64).amax(-1, keepdim=True)
        bound = U16 * ref.abs() + 8 * U32 * top
        if gamma is not None:
            clean = torch.where(torch.isfinite(x).all(-1, keepdim=True), x, torch.zeros_like(x))
            bound = _ref(clean, gamma, cos, sin, pos, inter)[1]             # (beside infinity: 0, exactly; beside NaN: NaN)
        within(got, ref, bound, (form, inter, norm))
        if gamma is None:
            past, held = x[..., rot:], got[..., rot:]
            assert torch.equal(torch.isnan(past), torch.isnan(held)) and torch.equal(past[~torch.isnan(past)], held[~torch.isnan(past)])
        return ref

    close(out, q, gq)
    hk, _, ke, _ = _held(cache, slots)
    if form == "bf16":
        close(hk, k, gk)
        return
    ref, _ = _ref(k, gk, cos, sin, pos, inter)
    if form == "fp4":
        rc, re = quantised4(ref)
        assert torch.equal(ke, re) and torch.equal(widened4(hk, ke)[ke.repeat_interleave(32, -1) != 255], widened4(rc, re)[re.repeat_interleave(32, -1) != 255])
        return
    fine = torch.isfinite(ref)
    x = torch.where(fine, ref, torch.zeros_like(ref))
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0)), torch.zeros_like(top)).clamp(min=-117)
    a = x / torch.exp2(e)[..., None]
    step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
    codes = hk.view(torch.float8_e4m3fn).to(F64)
    assert torch.equal(ke.to(F64), e + 127)
    assert torch.equal(torch.isnan(codes), ~fine) and torch.equal(codes[fine], (torch.round(a / step) * step)[fine])
