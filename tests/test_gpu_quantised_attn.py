"""Attention over a 4-bit paged cache against the 64-bit form: lengths from one token, ragged batches, every grouping of heads and kernel form, windows, rows that see
nothing, and anything at all in the cache behind a sequence's end."""
import pytest
import torch

from paper_2510_00206_amd import binding
from quant_util import widened4
from serve_util import BF16, F64, attention, gen, normal, within

pytestmark = pytest.mark.gpu


def _setup(seqs, H, G, D, page, seed, junk=True, spare=3, std=1.0):
    """seqs: [(new, length)].  (q, cache, table, offsets, lens, keys and values of each sequence in 64 bits)"""
    g = gen(seed)
    used = [-(-kv // page) for _, kv in seqs]
    pages = sum(used) + spare
    width = max(used + [1]) + 2
    codes = torch.randint(0, 256, (2, pages, G, page, D // 2), generator=g, dtype=torch.uint8)
    exps = torch.randint(123, 128, (2, pages, G, page, D // 32), generator=g, dtype=torch.uint8)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(seqs), width), 1 << 30 if junk else 0, dtype=torch.int32)
    table[:, 1::2] = -5 if junk else 0
    kd, vd = (widened4(codes[i], exps[i]) for i in range(2))
    at = 0
    for b, (_, kv) in enumerate(seqs):
        table[b, :used[b]] = order[at:at + used[b]]
        if kv % page and junk:
            exps[:, int(order[at + used[b] - 1]), :, kv % page:] = 255                # reads as NaN
        at += used[b]
    n = [a for a, _ in seqs]
    q = normal(g, (sum(n), H, D), std)
    offsets = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32)
    lens = torch.tensor([kv for _, kv in seqs], dtype=torch.int32)
    held = [tuple(x[table[b, :used[b]].long()].transpose(1, 2).reshape(-1, G, D)[:kv] for x in (kd, vd)) for b, (_, kv) in enumerate(seqs)]
    return q, binding.KVCache(codes[0].cuda(), codes[1].cuda(), exps[0].cuda(), exps[1].cuda()), table, offsets, lens, held


def _check(seqs, H, G, D, page, window=0, scale=None, seed=0, max_kv=None, std=1.0):
    print("attention over 4 bits", seqs[:4], len(seqs), H, G, D, page, window, flush=True)
    q, cache, table, offsets, lens, held = _setup(seqs, H, G, D, page, seed, std=std)
    out = torch.full(q.shape, 7.0, dtype=BF16, device="cuda")
    max_new = max([a for a, _ in seqs] + [1])
    binding.lora_paged_attn_fwd(q.cuda(), cache, table.cuda(), offsets.cuda(), lens.cuda(), max_new, max(max(kv for _, kv in seqs), 1) if max_kv is None else max_kv,
                                scale=scale, window=window, out=out)
    torch.cuda.synchronize()
    at = 0
    for b, (n, kv) in enumerate(seqs):
        ref, bound = attention(q[at:at + n].to(F64), *held[b], n, kv, D ** -0.5 if scale is None else scale, window)
        within(out[at:at + n], ref, bound + 1e-30, (b, n, kv, H, G, D, page, window))
        at += n


@pytest.mark.parametrize("H,G,D,page", [(8, 2, 64, 16), (4, 4, 128, 32), (7, 1, 128, 16), (24, 1, 64, 64), (40, 1, 128, 16), (32, 8, 128, 128), (3, 3, 64, 1024)])
def test_one_token(H, G, D, page):
    _check([(1, 1), (1, 2), (1, 15), (1, 16), (1, 17), (1, 33), (1, 100), (1, 257)], H, G, D, page, seed=H)


@pytest.mark.parametrize("H,G,D,page", [(8, 2, 64, 16), (2, 2, 128, 32), (3, 1, 128, 16), (16, 2, 64, 64), (6, 2, 128, 64)])
def test_chunks(H, G, D, page):
    _check([(1, 1), (5, 5), (7, 200), (64, 64), (33, 150), (70, 301)], H, G, D, page, seed=H + 1)


@pytest.mark.parametrize("n", [2, 8, 9, 16, 17, 31, 32, 33, 127, 128, 129, 200])
def test_rows_at_the_edges_of_the_tiles(n):
    _check([(n, n + 41), (n - 1, n + 90)], 2, 2, 64, 16, seed=n)
    _check([(n, n + 41)], 4, 2, 128, 16, seed=n)


@pytest.mark.parametrize("window", [1, 2, 16, 33, 64, 500, 10 ** 6])
@pytest.mark.parametrize("seqs", [[(1, 700), (1, 40), (1, 1)], [(5, 300), (9, 9)], [(90, 400), (150, 150)]])
def test_window(seqs, window):
    _check(seqs, 8, 2, 64, 16, window=window, seed=window)
    _check(seqs, 4, 2, 128, 32, window=window, seed=window)


def test_rows_that_see_nothing_and_empty_sequences():
    for H, G, D in ((8, 2, 64), (2, 2, 128), (40, 1, 64)):
        _check([(0, 0), (3, 1), (1, 0), (0, 50), (40, 7), (100, 20), (0, 0)], H, G, D, 16)
        _check([(3, 1), (200, 0), (60, 60)], H, G, D, 16, window=5)


@pytest.mark.parametrize("seqs,H,G,D,page", [
    ([(1, 5000)], 8, 2, 128, 16), ([(1, 3001), (1, 20), (1, 1500)], 4, 1, 64, 32), ([(4, 4099), (2, 100)], 16, 2, 128, 64),
    ([(70, 3000), (3, 2000)], 4, 2, 64, 16), ([(150, 2500)], 2, 1, 128, 16)])
def test_long_ranges_in_parts(seqs, H, G, D, page):
    _check(seqs, H, G, D, page, seed=5)
    _check(seqs, H, G, D, page, seed=6, max_kv=max(kv for _, kv in seqs) // 2)


@pytest.mark.parametrize("std", [30.0, 300.0])
def test_large_scores(std):
    _check([(1, 300), (9, 60)], 8, 2, 128, 16, std=std)
    _check([(90, 200)], 8, 2, 64, 16, std=std)


@pytest.mark.parametrize("seqs", [[(1, 40), (7, 50)], [(90, 200)]])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_in_places_that_a_row_does_not_see(seqs, D):
    """32 entries of keys or values that are NaN reach the rows that see their token (of values: in their columns) and no other."""
    H, G, page = 4, 2, 16
    q, cache, table, offsets, lens, held = _setup(seqs, H, G, D, page, 3)
    run = lambda: binding.lora_paged_attn_fwd(q.cuda(), cache, table.cuda(), offsets.cuda(), lens.cuda(), max(n for n, _ in seqs), max(k for _, k in seqs)).cpu()
    want, at = run(), int(offsets[len(seqs) - 1])
    n, kv = seqs[-1]
    token = kv - n // 2                                                 # the first n - n // 2 rows of the sequence do not see it
    first = at + token - (kv - n)
    pg, o = int(table[len(seqs) - 1, token // page]), token % page
    cache.tensors[3][pg, 0, o, 1] = 255
    got = run()
    bad = ~torch.isfinite(got)
    hit = torch.zeros_like(bad)
    hit[first:at + n, :H // G, 32:64] = True
    assert torch.equal(bad, hit) and torch.equal(got[~hit], want[~hit])
    cache.tensors[2][pg, 1, o, D // 32 - 1] = 255
    hit[first:at + n, H // G:] = True
    got = run()
    assert torch.equal(~torch.isfinite(got), hit) and torch.equal(got[~hit], want[~hit])


def test_one_workspace_for_smaller_steps():
    seqs, H, G, D, page = [(1, 3000), (1, 700), (1, 20)], 8, 2, 128, 16
    q, cache, table, offsets, lens, held = _setup(seqs, H, G, D, page, 2)
    ws = binding.alloc_paged_attn_workspace(cache, 3, H, 3, 1, 3000)
    ws.fill_(0xFF)
    out = binding.lora_paged_attn_fwd(q.cuda(), cache, table.cuda(), offsets.cuda(), lens.cuda(), 1, 3000, workspace=ws).cpu()
    one = binding.lora_paged_attn_fwd(q[:1].cuda(), cache, table[:1].cuda(), offsets[:2].cuda(), lens[:1].cuda(), 1, 3000, workspace=ws).cpu()
    for got, b in ((out[0:1], 0), (out[1:2], 1), (out[2:3], 2), (one, 0)):
        ref, bound = attention(q[b:b + 1].to(F64), *held[b], 1, seqs[b][1], D ** -0.5, 0)
        within(got, ref, bound + 1e-30, b)


def test_a_cache_past_2_to_32_bytes():
    """Pages whose first byte lies past 2^32, and exponents past 2^31 bytes of codes."""
    H, G, D, page, pages = 8, 8, 128, 64, 140000                        # 4.6 GB of keys
    k = torch.zeros((pages, G, page, D // 2), dtype=torch.uint8, device="cuda")
    e = torch.full((pages, G, page, D // 32), 127, dtype=torch.uint8, device="cuda")
    assert k.numel() > 1 << 32
    g = gen(7)
    at = [pages - 1, 3, pages - 2, 70000]
    codes = torch.randint(0, 256, (4, G, page, D // 2), generator=g, dtype=torch.uint8)
    for i, p in enumerate(at):
        k[p] = codes[i].cuda()
    cache = binding.KVCache(k, k, e, e)
    table, kv = torch.tensor([at], dtype=torch.int32), 4 * page - 5
    held = widened4(codes, torch.full((4, G, page, D // 32), 127, dtype=torch.uint8)).transpose(1, 2).reshape(-1, G, D)[:kv]
    for n in (1, 40):
        q = normal(g, (n, H, D), 0.2)
        out = binding.lora_paged_attn_fwd(q.cuda(), cache, table.cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([kv], dtype=torch.int32).cuda(), n, kv)
        ref, bound = attention(q.to(F64), held, held, n, kv, D ** -0.5, 0)
        within(out, ref, bound + 1e-30, n)
    slots = torch.tensor([p * page + 17 for p in at], device="cuda")
    back, _ = binding.lora_kv_cache_read(cache, slots)
    assert torch.equal(back.cpu().to(F64), widened4(codes[:, :, 17], torch.full((4, G, D // 32), 127, dtype=torch.uint8)))
    new = normal(g, (4, G, D))
    cos, sin = torch.ones((1, D // 2), device="cuda"), torch.zeros((1, D // 2), device="cuda")
    binding.lora_kv_cache_append(cache, new.cuda(), new.cuda(), new.cuda(), cos, sin, torch.zeros(4, dtype=torch.int32, device="cuda"), slots)
    a, _ = binding.lora_kv_cache_read(cache, slots)
    binding.lora_kv_cache_write(cache, new.cuda(), new.cuda(), slots)
    b, _ = binding.lora_kv_cache_read(cache, slots)
    assert torch.equal(a, b)
