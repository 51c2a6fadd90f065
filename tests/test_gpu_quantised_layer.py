"""The LoRA layer of many requests over 4-bit weights against the 64-bit form: one row to many, adapters in any order, none, of any rank, no adapters at all."""
import pytest
import torch

from paper_2510_00206_amd import binding
from quant_util import WRAPPED, quantised4, widened4
from serve_util import BF16, U32, U16, F64, gen, normal, requests, within

pytestmark = pytest.mark.gpu


def _weights(g, N, K):
    codes, exps = quantised4(normal(g, (N, K), K ** -0.5))
    return codes, exps


def _case(M, K, N, r, P, ids, mixed, seed, scale_b=0.1):
    g = gen(seed)
    X = normal(g, (M, K))
    codes, exps = _weights(g, N, K)
    A, B = normal(g, (P, r, K), K ** -0.5), normal(g, (P, N, r), scale_b)
    s = torch.rand(P, generator=g) * 2 - 0.5
    ranks = torch.randint(0, r + 1, (P,), generator=g, dtype=torch.int32) if mixed else None
    if ids == "each":
        ids = torch.randperm(max(M, P), generator=g)[:M] % P
    elif ids == "chunks":
        ids = torch.arange(M) * 3 // max(M, 1) % P
    elif ids == "none":
        ids = torch.full((M,), -1)
    else:
        ids = torch.randint(-1, P, (M,), generator=g)
    return X, codes, exps, A, B, ids.to(torch.int32), s, ranks


def _check(case, label):
    print("layer over 4 bits", label, flush=True)
    X, codes, exps, A, B, ids, s, ranks = case
    dev = [t.cuda() for t in (X, codes, exps, A, B, ids, s)]
    Y, S = torch.full((X.shape[0], codes.shape[0]), 7.0, dtype=BF16, device="cuda"), torch.full((X.shape[0], A.shape[1]), 7.0, dtype=BF16, device="cuda")
    binding.lora_requests_quantised_fwd(*dev, ranks=None if ranks is None else ranks.cuda(), Y=Y, S=S)
    torch.cuda.synchronize()
    ref, bound, sref, sbound = requests(X, widened4(codes, exps), A, B, ids, s, ranks)
    within(S, sref, sbound, (label, "S"))
    within(Y, ref, bound, (label, "Y"))
    return Y


@pytest.mark.parametrize("M,K,N,r,P,ids,mixed", [
    (1, 64, 64, 16, 1, "any", False),               # half a block of the contraction
    (1, 1024, 192, 64, 5, "any", True),
    (2, 576, 320, 32, 3, "each", False),
    (15, 128, 64, 16, 2, "any", False),
    (16, 4096, 128, 64, 9, "each", True),
    (17, 256, 128, 16, 40, "each", True),           # a block of 16 rows and one more, an adapter to every row
    (32, 192, 64, 32, 3, "any", True),
    (33, 64, 448, 64, 33, "each", False),
    (48, 320, 64, 16, 3, "chunks", False),
    (64, 4096, 256, 16, 48, "any", False),
    (65, 448, 1088, 32, 7, "any", True),
    (129, 320, 576, 64, 200, "each", True),
    (200, 192, 4160, 16, 3, "chunks", False),
    (300, 512, 64, 32, 2, "none", False),
    (511, 128, 320, 64, 9, "chunks", True),
    (777, 64, 1024, 32, 5, "any", True),
    (3, 14336, 128, 16, 3, "any", False),
])
def test_against_64_bits(M, K, N, r, P, ids, mixed):
    _check(_case(M, K, N, r, P, ids, mixed, 100 + M), (M, K, N, r, P, ids))


@pytest.mark.parametrize("M,K,N", [(1024, 512, 4096), (1300, 256, 4096), (2100, 192, 2112), (600, 128, 14336), (257, 1024, 6144), (100, 256, 8192), (40, 128, 16448)])
def test_large(M, K, N):
    _check(_case(M, K, N, 32, 11, "chunks", True, M), (M, K, N))


@pytest.mark.parametrize("M,K,N", [(1, 64, 64), (5, 4096, 4096), (31, 1088, 128), (64, 256, 192), (100, 128, 1024), (500, 320, 2048), (1500, 192, 640)])
def test_without_adapters(M, K, N):
    g = gen(M)
    X, (codes, exps) = normal(g, (M, K)), _weights(g, N, K)
    Y, S = binding.lora_requests_quantised_fwd(X.cuda(), codes.cuda(), exps.cuda())
    assert S is None
    W = widened4(codes, exps)
    ref = X.to(F64) @ W.t()
    within(Y, ref, U16 * ref.abs() + (1 + U16) * K * U32 * (X.to(F64).abs() @ W.abs().t()), (M, K, N))


@pytest.mark.parametrize("M", [1, 20, 40, 140, 600])
def test_padding_and_foreign_ids(M):
    """Rows and columns past an adapter's rank hold anything; ids outside the pool have no adapter."""
    K, N, r, P = 192, 256, 32, 4
    X, codes, exps, A, B, ids, s, ranks = _case(M, K, N, r, P, "any", True, M)
    ranks = torch.tensor([5, 32, 0, 17], dtype=torch.int32)
    for g in range(P):
        A[g, int(ranks[g]):], B[g, :, int(ranks[g]):] = float("nan"), float("inf")
    ids[::3] = torch.tensor([P, P + 7, -9, 1 << 30, -(1 << 31)], dtype=torch.int32).repeat(M)[:ids[::3].numel()]
    _check((X, codes, exps, A, B, ids, s, ranks), ("padding", M))


@pytest.mark.parametrize("M", [4, 40, 300])
def test_what_is_not_finite_stays_in_its_place(M):
    """NaN and infinities of a row of X stay in its row of Y, those of 32 weights (held as NaN) in their column, those of an adapter with its rows."""
    K, N = 320, 192
    X, codes, exps, A, B, ids, s, _ = _case(M, K, N, 16, 3, "any", False, M)
    ids[0], ids[1], ids[2], ids[3] = 1, 0, -1, 2
    ref = _check((X, codes, exps, A, B, ids, s, None), ("finite", M)).cpu()
    X2, e2, B2 = X.clone(), exps.clone(), B.clone()
    X2[1, K - 1] = float("nan")                      # in the half block at the contraction's end
    X2[3, 5] = float("inf")
    e2[7, K // 32 - 1] = 255
    B2[1, 9, 3] = float("inf")
    Y, _ = binding.lora_requests_quantised_fwd(X2.cuda(), codes.cuda(), e2.cuda(), A.cuda(), B2.cuda(), ids.cuda(), s.cuda())
    Y = Y.cpu()
    bad = ~torch.isfinite(Y)
    assert bool(bad[1].all()) and bool(torch.isnan(Y[:, 7]).all())
    hit = torch.zeros_like(bad)
    hit[1], hit[3], hit[:, 7] = True, True, True
    hit[ids == 1, 9] = True
    assert not bool(bad[~hit].any()) and torch.equal(Y[~hit], ref[~hit])
    assert bool(bad[(ids == 1).nonzero()[:, 0], 9].all())


def test_the_same_bits_again_and_in_any_batch():
    """The same call gives the same bits; rows past the batch are not touched."""
    X, codes, exps, A, B, ids, s, ranks = (None if t is None else t.cuda() for t in _case(90, 512, 320, 32, 6, "any", True, 3))
    Y = torch.full((100, 320), 7.0, dtype=BF16, device="cuda")
    a, _ = binding.lora_requests_quantised_fwd(X, codes, exps, A, B, ids, s, ranks=ranks, Y=Y[:90])
    one = a.clone()
    for _ in range(3):
        binding.lora_requests_quantised_fwd(X, codes, exps, A, B, ids, s, ranks=ranks, Y=Y[:90])
        assert torch.equal(Y[:90], one)
    assert bool((Y[90:] == 7.0).all())


def test_large_offsets():
    """Weights whose codes pass 2^31 bytes, at their ends."""
    N, K, M = 1 << 20, 4160, 3
    codes = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    exps = torch.full((N, K // 32), 127, dtype=torch.uint8, device="cuda")
    g = gen(1)
    X = normal(g, (M, K))
    last = torch.randint(0, 256, (64, K // 2), generator=g, dtype=torch.uint8)
    codes[-64:] = last.cuda()
    Y, _ = binding.lora_requests_quantised_fwd(X.cuda(), codes, exps)
    W = widened4(last, torch.full((64, K // 32), 127, dtype=torch.uint8))
    ref = X.to(F64) @ W.t()
    within(Y[:, -64:], ref, U16 * ref.abs() + (1 + U16) * K * U32 * (X.to(F64).abs() @ W.abs().t()), "last rows")
    assert int((Y[:, :-64] != 0).sum()) == 0
    W = binding.lora_weights_read(codes, exps)
    assert torch.equal(W[-64:].cpu().to(F64), widened4(last, torch.full((64, K // 32), 127, dtype=torch.uint8)))
    c2, e2 = binding.lora_weights_write(W)
    assert torch.equal(binding.lora_weights_read(c2, e2)[-64:], W[-64:])


@pytest.mark.parametrize("P", [0, 5])
@pytest.mark.parametrize("M,K,N", [
    (3, 192, 64), (4, 256, 4096),                          # 16 x 16 with four rows at most
    (5, 256, 128), (16, 192, 4096),                        # 16 x 16
    (16, 192, 6144), (20, 256, 4096),                      # 16 x 32
    (30, 256, 4160), (16, 192, 8960),                      # 16 x 64
    (48, 192, 6144), (96, 320, 4096), (40, 512, 8192),     # 32 x 64
    (130, 192, 4160), (129, 256, 4160),                    # 64 x 64
    (200, 192, 4160), (700, 256, 2112),                    # 64 x 128
    (260, 256, 8192), (600, 192, 4096),                    # 64 x 256
    (1300, 256, 4096), (2050, 320, 2112),                  # 128 x 256
])
def test_every_tile(M, K, N, P):
    """Contractions that end with a block of 128 and with half a one, rows and columns past the last tile, with and without adapters."""
    if P:
        _check(_case(M, K, N, 16, P, "any", True, M + K), (M, K, N, P))
    else:
        test_without_adapters(M, K, N)


def test_most_rows():
    """2^21 - 1 rows, each an adapter of its own choice: the first and the last ones."""
    M, K, N, r, P = (1 << 21) - 1, 64, 64, 16, 3
    X, codes, exps, A, B, ids, s, _ = _case(600, K, N, r, P, "any", False, 5)
    big = torch.zeros((M, K), dtype=BF16, device="cuda")
    far = torch.full((M,), -1, dtype=torch.int32, device="cuda")
    big[:300], big[-300:], far[:300], far[-300:] = X[:300].cuda(), X[300:].cuda(), ids[:300].cuda(), ids[300:].cuda()
    Y, _ = binding.lora_requests_quantised_fwd(big, codes.cuda(), exps.cuda(), A.cuda(), B.cuda(), far, s.cuda())
    ref, bound, _, _ = requests(X, widened4(codes, exps), A, B, ids, s, None)
    within(Y[:300], ref[:300], bound[:300], "first rows")
    within(Y[-300:], ref[300:], bound[300:], "last rows")
    assert int((Y[300:-300] != 0).sum()) == 0


@pytest.mark.parametrize("M,K,N,r,ids,mixed", [
    (1, 64, 64, 16, "any", False), (1, 4096, 192, 16, "any", True), (1, 1024, 4096, 32, "any", True), (1, 192, 128, 64, "any", True), (1, 256, 64, 64, "each", False),
    (2, 1024, 320, 16, "each", True), (2, 64, 64, 64, "each", True), (3, 320, 256, 16, "any", True), (4, 256, 128, 16, "each", True), (4, 64, 64, 32, "none", False),
    (1, 4160, 192, 16, "any", True), (4, 320, 64, 16, "each", False)])                     # (the last two: S from a launch of its own)
def test_a_few_rows_in_one_launch(M, K, N, r, ids, mixed):
    """S formed beside the base product: every row with an adapter of its own rank, S as it is returned too, what is past a rank anything."""
    for seed in range(4):
        X, codes, exps, A, B, i, s, ranks = _case(M, K, N, r, 5, ids, mixed, seed)
        if seed and ids != "none":
            i = (torch.arange(M) + seed).to(torch.int32) % 5
        if mixed:
            ranks = torch.tensor([0, 1, r - 1, r // 2, r], dtype=torch.int32)[torch.randperm(5, generator=gen(seed))]
            for g in range(5):
                A[g, int(ranks[g]):], B[g, :, int(ranks[g]):] = float("nan"), float("inf")
        _check((X, codes, exps, A, B, i, s, ranks), ("one launch", M, K, N, r, seed))


def test_an_adapter_that_diverged_in_one_launch():
    X, codes, exps, A, B, ids, s, _ = _case(3, 128, 192, 16, 3, "any", False, 9)
    ids[:] = torch.tensor([0, 1, -1])
    want = _check((X, codes, exps, A, B, ids, s, None), "diverged").cpu()
    B[1, 7, 3], A[2, 5, 5], B[2] = float("inf"), float("nan"), float("nan")
    Y, _ = binding.lora_requests_quantised_fwd(*(t.cuda() for t in (X, codes, exps, A, B, ids, s)))
    bad = ~torch.isfinite(Y.cpu())
    assert bool(bad[1, 7]) and int(bad.sum()) == 1 and torch.equal(Y.cpu()[~bad], want[~bad])


@pytest.mark.parametrize("P", [0, 5])
@pytest.mark.parametrize("tile,M,K,N", WRAPPED)
def test_rings_that_wrap(tile, M, K, N, P):
    """Every kind of tile over contractions of more than twice what its rings hold, so that every place is filled again and again and the waits are counted ones."""
    t = binding.lora_debug_quantised_tiles(M, K, N, 32, P)
    assert (t.rows, t.columns) == tile and K // 128 > 2 * t.ring_blocks
    g = gen(M + K)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, dtype=torch.uint8)
    exps = torch.randint(118, 123, (N, K // 32), generator=g, dtype=torch.uint8)
    X = normal(g, (M, K))
    if P:
        A, B, s = normal(g, (P, 32, K), K ** -0.5), normal(g, (P, N, 32), 0.1), torch.rand(P, generator=g) * 2 - 0.5
        ids, ranks = torch.randint(-1, P, (M,), generator=g, dtype=torch.int32), torch.randint(0, 33, (P,), generator=g, dtype=torch.int32)
        _check((X, codes, exps, A, B, ids, s, ranks), ("wrapped", tile, M, K, N))
        return
    print("wrapped, no adapters", tile, M, K, N, flush=True)
    Y, _ = binding.lora_requests_quantised_fwd(X.cuda(), codes.cuda(), exps.cuda())
    W = widened4(codes, exps)
    ref = X.to(F64) @ W.t()
    within(Y, ref, U16 * ref.abs() + (1 + U16) * K * U32 * (X.to(F64).abs() @ W.abs().t()), (tile, M, K, N))
