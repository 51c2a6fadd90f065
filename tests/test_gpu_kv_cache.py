"""The paged cache: codes, exponents and what is read back, bit for bit."""
import pytest
import torch

from paper_2510_00206_amd import binding
from serve_util import BF16, gen, normal, quantised, widened

pytestmark = pytest.mark.gpu


def _slots(g, pages, page, M):
    return torch.randperm(pages * page, generator=g)[:M]


@pytest.mark.parametrize("M,G,D,page,fp8", [(1, 1, 16, 16, True), (1, 8, 128, 16, False), (5, 3, 64, 32, True), (37, 2, 80, 64, True), (100, 8, 128, 16, True),
                                            (33, 1, 256, 128, True), (64, 4, 208, 16, False), (50, 5, 48, 1024, True)])
def test_write_and_read(M, G, D, page, fp8):
    print("cache", M, G, D, page, fp8, flush=True)
    g = gen(M + D)
    pages = M // page + 2
    spread = torch.exp2(torch.randint(-60, 60, (M, G, 1), generator=g).float())
    kv = torch.stack((normal(g, (M, G, D)).float() * spread, normal(g, (M, G, D)).float() / spread), 1).to(BF16)
    kv[0, 0, 0] = 0                                                     # a head of zeros
    kv[0, 1, 0, :2] = torch.tensor([float("inf"), -float("inf")])
    kv[M - 1, 0, G - 1, 3] = float("nan")
    kv[M - 1, 1, G - 1] = normal(g, (D,)).float() * 2.0 ** -130         # below what a scale reaches
    slots = _slots(g, pages, page, M)
    cache = binding.KVCache.empty(pages, page, G, D, fp8)
    for t in cache.tensors:
        if t is not None:
            t.view(torch.uint8).fill_(0x11)
    dev = kv.cuda()
    binding.lora_kv_cache_write(cache, dev[:, 0], dev[:, 1], slots.cuda())
    p, o = slots // page, slots % page
    left = torch.ones((pages, page), dtype=torch.bool)
    left[p, o] = False
    back = binding.lora_kv_cache_read(cache, slots.cuda())
    for i in range(2):
        held, x = cache.tensors[i].cpu(), kv[:, i]
        if not fp8:
            assert torch.equal(held[p, :, o].view(torch.int16), x.contiguous().view(torch.int16))
            assert torch.equal(back[i].cpu().view(torch.int16), x.contiguous().view(torch.int16))
            continue
        codes, exps = quantised(x)
        got = held.view(torch.uint8)[p, :, o]
        nan = (codes & 0x7F) == 0x7F
        assert torch.equal((got & 0x7F) == 0x7F, nan) and torch.equal(got[~nan], codes[~nan])
        assert torch.equal(cache.tensors[2 + i].cpu()[p, :, o], exps)
        want = widened(codes, exps)
        assert torch.equal(torch.isnan(back[i].cpu()), nan) and torch.equal(back[i].cpu().double()[~nan], want[~nan])
        assert bool((held.view(torch.uint8).transpose(1, 2)[left] == 0x11).all()) and bool((cache.tensors[2 + i].cpu().transpose(1, 2)[left] == 0x11).all())


def test_every_code():
    """All 256 codes read back as their values, and written again give themselves (NaN: one of the two)."""
    cache = binding.KVCache.empty(2, 16, 1, 256, True)
    k, v, ke, ve = cache.tensors
    k.view(torch.uint8)[:] = torch.arange(256, dtype=torch.uint8, device="cuda")
    exps = torch.arange(10, 248, 8, dtype=torch.uint8)[:30]
    ke.view(-1)[:30] = exps.cuda()
    slots = torch.arange(30, device="cuda")
    got, _ = binding.lora_kv_cache_read(cache, slots)
    codes = torch.arange(256, dtype=torch.uint8).expand(30, 256).contiguous()
    want = widened(codes, exps)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got[:, 0].cpu()), nan) and torch.equal(got[:, 0].cpu().double()[~nan], want[~nan])
    other = binding.KVCache.empty(2, 16, 1, 256, True)
    binding.lora_kv_cache_write(other, got, got, slots)
    assert torch.equal(other.tensors[0].view(torch.uint8).view(32, 256)[:30].cpu()[~nan], codes[~nan])
    assert torch.equal(other.tensors[2].view(-1)[:30].cpu(), exps)


def test_rounding_and_the_scale_at_its_steps():
    """Magnitudes on both sides of 448 x 2^e, and values half-way between two codes, which go to the even one."""
    rows = []
    for top in (1.75, 1.7578125, 1.9921875, 1.0, 0.99609375, 448.0, 450.0):
        r = torch.zeros(64)
        r[0] = top
        r[1:] = torch.arange(63).float() * top / 64
        rows.append(r)
    x = torch.stack(rows).to(BF16)[:, None]
    cache = binding.KVCache.empty(1, 16, 1, 64, True)
    binding.lora_kv_cache_write(cache, x.cuda(), (-x).cuda(), torch.arange(len(rows)).cuda())
    for i, y in enumerate((x, -x)):
        codes, exps = quantised(y)
        assert torch.equal(cache.tensors[2 + i].cpu()[0, 0, :len(rows)], exps[:, 0])
        assert torch.equal(cache.tensors[i].view(torch.uint8).cpu()[0, 0, :len(rows)], codes[:, 0])


def test_slots_outside_the_cache():
    for fp8 in (True, False):
        cache = binding.KVCache.empty(3, 16, 2, 64, fp8)
        x = normal(gen(1), (6, 2, 64)).cuda()
        slots = torch.tensor([-1, 5, 48, 1 << 40, -(1 << 62), 47], device="cuda")
        binding.lora_kv_cache_write(cache, x, x, slots)
        for t in cache.tensors[:2]:
            rows = t.float().transpose(1, 2).reshape(48, -1).abs().sum(1).nonzero()[:, 0].tolist()
            assert rows == [5, 47]
        k, v = binding.lora_kv_cache_read(cache, slots)
        assert not k[[0, 2, 3, 4]].any() and bool(k[[1, 5]].any(-1).all()) and torch.equal(k, v)


def test_cache_past_32_bits():
    """The last slots of a cache of more than 2^32 bytes and 2^31 elements a side."""
    for fp8 in (True, False):
        pages, page, G, D = (1 << 31) // (64 * 8 * 128) + 3, 64, 8, 128
        cache = binding.KVCache.empty(pages, page, G, D, fp8)
        x = normal(gen(2), (3, G, D))
        slots = torch.tensor([0, pages * page - 1, pages * page - 65], device="cuda")
        binding.lora_kv_cache_write(cache, x.cuda(), (-x).cuda(), slots)
        k, v = binding.lora_kv_cache_read(cache, slots)
        want = widened(*quantised(x)) if fp8 else x.double()
        assert torch.equal(k.cpu().double(), want) and torch.equal(v.cpu().double(), -want)
        del cache


def test_no_rows_and_arguments():
    cache = binding.KVCache.empty(2, 16, 2, 64, True)
    x, slots = normal(gen(1), (4, 2, 64)).cuda(), torch.arange(4, device="cuda")
    binding.lora_kv_cache_write(cache, x[:0], x[:0], slots[:0])
    assert binding.lora_kv_cache_read(cache, slots[:0])[0].shape == (0, 2, 64)
    for bad in ((x.float(), x, slots), (x, x, slots.int()), (x, x[:2], slots), (x[:, :1], x[:, :1], slots), (x, x, slots[:3])):
        with pytest.raises(AssertionError):
            binding.lora_kv_cache_write(cache, *bad)
    k, v, ke, ve = cache.tensors
    for bad in ((k, v), (k, v, ke), (k, v.to(BF16), ke, ve), (k.float(), v.float()), (k[0], v[0], ke, ve), (k, v, ke[:1], ve)):
        with pytest.raises(AssertionError):
            binding.KVCache(*bad)


@pytest.mark.parametrize("M,G,D,fp8", [(16500, 8, 128, True), (16500, 8, 128, False), (33000, 8, 64, True), (8300, 8, 256, True), (8300, 8, 208, False)])
def test_large_reads(M, G, D, fp8):
    """Outputs of more than 64 MB, which go past the caches, are those of reads of a thousand tokens (and, in bf16, what was written)."""
    print("large reads", M, G, D, fp8, flush=True)
    if D == 208:
        M = 10200
    page = 16
    cache = binding.KVCache.empty(M // page + 1, page, G, D, fp8)
    kv = torch.randn((M, 2, G, D), device="cuda").to(BF16)
    slots = torch.randperm(M // page * page + page, device="cuda")[:M]
    slots[5] = -1
    binding.lora_kv_cache_write(cache, kv[:, 0], kv[:, 1], slots)
    whole = binding.lora_kv_cache_read(cache, slots)
    assert 2 * whole[0].numel() * 2 >= 64 << 20
    for i in range(2):
        for at in range(0, M, 1000):
            piece = binding.lora_kv_cache_read(cache, slots[at:at + 1000])[i]
            assert torch.equal(whole[i][at:at + 1000], piece)
        assert not whole[i][5].any()
        if not fp8:
            kv[5] = 0
            assert torch.equal(whole[i], kv[:, i])


@pytest.mark.parametrize("fp8", [True, False])
def test_a_slot_that_two_rows_name(fp8):
    """Undefined in itself, and without effect on any other slot."""
    cache = binding.KVCache.empty(4, 16, 3, 128, fp8)
    x = normal(gen(4), (40, 3, 128))
    slots = torch.arange(40) + 10
    slots[20:30] = 12
    binding.lora_kv_cache_write(cache, x.cuda(), (-x).cuda(), slots.cuda())
    single = torch.tensor([i for i in range(40) if slots[i] != 12])
    k, v = binding.lora_kv_cache_read(cache, slots[single].cuda())
    want = widened(*quantised(x[single])) if fp8 else x[single].double()
    assert torch.equal(k.cpu().double(), want) and torch.equal(v.cpu().double(), -want)
    others = torch.tensor([i for i in range(64) if i not in slots.tolist()])
    k, v = binding.lora_kv_cache_read(cache, others.cuda())
    assert not k.any() and not v.any()


@pytest.mark.parametrize("M,G,D,fp8", [(46000, 8, 128, True), (46001, 8, 128, False), (92000, 8, 64, True), (23003, 8, 256, True), (185000, 2, 80, False)])
def test_larger_reads(M, G, D, fp8):
    """Outputs on both sides of the size from which they go past the caches."""
    page = 16
    cache = binding.KVCache.empty(M // page + 1, page, G, D, fp8)
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    kv = torch.randn((M, 2, G, D), generator=g, device="cuda").to(BF16)
    slots = torch.randperm(M // page * page + page, generator=g, device="cuda")[:M]
    binding.lora_kv_cache_write(cache, kv[:, 0], kv[:, 1], slots)
    slots[77] = -1
    whole = binding.lora_kv_cache_read(cache, slots)
    assert 4 * whole[0].numel() >= 176 << 20 or D == 80
    pieces = [binding.lora_kv_cache_read(cache, part.contiguous()) for part in slots.split(4001)]
    for i in range(2):
        assert torch.equal(whole[i], torch.cat([p[i] for p in pieces])) and not whole[i][77].any()
        if not fp8:
            kv[77] = 0
            assert torch.equal(whole[i], kv[:, i])
