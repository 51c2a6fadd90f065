"""The LoRA linear layer of many requests against the 64-bit form: one row to more than one launch's worth, adapters in any order, none, of any rank,
with anything in the padding."""
import pytest
import torch

from paper_2510_00206_amd import binding
from serve_util import BF16, F32, U16, U32, gen, normal, requests, within

pytestmark = pytest.mark.gpu


def _case(M, K, N, r, P, ids, mixed, seed, scale_b=0.1):
    g = gen(seed)
    X, W = normal(g, (M, K)), normal(g, (N, K), K ** -0.5)
    A, B = normal(g, (P, r, K), K ** -0.5), normal(g, (P, N, r), scale_b)
    s = torch.rand(P, generator=g) * 2 - 0.5
    ranks = torch.randint(0, r + 1, (P,), generator=g, dtype=torch.int32) if mixed else None
    if ids == "each":
        ids = torch.randperm(max(M, P), generator=g)[:M] % P
    elif ids == "chunks":
        ids = torch.arange(M) * 3 // max(M, 1) % P
    elif ids == "one":
        ids = torch.full((M,), P - 1)
    elif ids == "none":
        ids = torch.full((M,), -1)
    else:
        ids = torch.randint(-1, P, (M,), generator=g)
    return X, W, A, B, ids.to(torch.int32), s, ranks


def _check(case, label):
    print("requests", label, flush=True)
    X, W, A, B, ids, s, ranks = case
    dev = [None if t is None else t.cuda() for t in (X, W, A, B, ids, s)]
    Y, S = torch.full((X.shape[0], W.shape[0]), 7.0, dtype=BF16, device="cuda"), torch.full((X.shape[0], A.shape[1]), 7.0, dtype=BF16, device="cuda")
    binding.lora_requests_fwd(*dev, ranks=None if ranks is None else ranks.cuda(), Y=Y, S=S)
    torch.cuda.synchronize()
    ref, bound, sref, sbound = requests(X, W, A, B, ids, s, ranks)
    within(S, sref, sbound, (label, "S"))
    within(Y, ref, bound, (label, "Y"))


@pytest.mark.parametrize("M,K,N,r,P,ids,mixed", [
    (1, 64, 64, 16, 1, "one", False),
    (1, 1024, 192, 64, 5, "any", True),
    (2, 576, 320, 32, 3, "each", False),
    (17, 256, 128, 16, 40, "each", True),           # a block of 16 rows and one more, an adapter to every row
    (33, 64, 448, 64, 33, "each", False),
    (64, 4096, 256, 16, 48, "any", False),          # half tiles, long contraction
    (100, 448, 1088, 32, 7, "any", True),
    (129, 320, 576, 64, 200, "each", True),         # four rows to a wave in the first product
    (200, 192, 4160, 16, 3, "chunks", False),
    (300, 512, 64, 32, 2, "none", False),
    (511, 128, 320, 64, 9, "chunks", True),
    (513, 320, 192, 16, 4, "chunks", True),         # 16 rows to a workgroup in the first product
    (530, 640, 256, 64, 530, "each", False),
    (777, 64, 1024, 32, 5, "any", True),
])
def test_against_64_bits(M, K, N, r, P, ids, mixed):
    _check(_case(M, K, N, r, P, ids, mixed, 100 + M), (M, K, N, r, P, ids))


@pytest.mark.parametrize("M,K,N", [(1024, 512, 4096), (1300, 256, 4096), (2100, 192, 2112), (600, 128, 14336)])
def test_large_tiles(M, K, N):
    """Rows enough for every tile of the GEMM family, and for two launches."""
    _check(_case(M, K, N, 32, 11, "chunks", True, M), (M, K, N))


@pytest.mark.parametrize("M", [5, 140, 600])
def test_padding_and_foreign_ids(M):
    """What lies past an adapter's rank, and the whole of adapters that no row names, may hold anything; ids outside the pool have no adapter."""
    X, W, A, B, ids, s, _ = _case(M, 256, 192, 32, 6, "any", False, M)
    ranks = torch.tensor([0, 5, 32, 16, 31, 99], dtype=torch.int32)
    ids[ids == 2] = 1
    ids[0], ids[M // 2], ids[M - 1] = 6, -7, 1 << 30
    for g in range(6):
        q = min(int(ranks[g]), 32)
        A[g, q:], B[g, :, q:] = float("nan"), float("inf")
    A[2], B[2], s[2] = float("nan"), float("nan"), float("nan")
    _check((X, W, A, B, ids, s, ranks), ("padding", M))


def test_not_finite_stays_with_its_row():
    """A request's not-finite input, and a diverged adapter, reach the rows that have them and no other."""
    for M in (20, 150, 600):
        X, W, A, B, ids, s, _ = _case(M, 128, 128, 16, 8, "any", False, M)
        ids[:] = torch.arange(M) % 7
        X[3, 5], A[4, 2, 7] = float("inf"), float("nan")
        Y, S = binding.lora_requests_fwd(*(t.cuda() for t in (X, W, A, B, ids, s)))
        bad = (~torch.isfinite(Y)).any(1).cpu()
        want = (ids == 4)
        want[3] = True
        assert torch.equal(bad, want), M


@pytest.mark.parametrize("r", [16, 32, 64])
@pytest.mark.parametrize("M,N", [(3, 192), (40, 6144), (70, 256), (200, 8192), (600, 4096), (1100, 4096)])
def test_diverged_second_factor(M, N, r):
    """Infinities and NaN in an adapter's B reach the columns of its own rows and nothing else: neither the other rows of a tile nor those without."""
    X, W, A, B, ids, s, _ = _case(M, 128, N, r, 8, "any", False, M + r)
    ids[:] = torch.arange(M) % 9 - 1
    B[2, 5, 3], B[2, 50, r - 1], B[5, N - 1, 0], B[5, 64, r // 2] = float("inf"), float("nan"), -float("inf"), float("nan")
    _check((X, W, A, B, ids, s, None), ("diverged", M, N, r))


def test_equals_the_layer_of_one_adapter():
    """All rows with one adapter: the forward of the training layer without dropout, up to the order of the sums in S."""
    X, W, A, B, ids, s, _ = _case(384, 512, 256, 32, 3, "one", False, 1)
    Y, S = binding.lora_requests_fwd(*(t.cuda() for t in (X, W, A, B, ids, s)))
    Y1, S1 = binding.lora_fwd(X.cuda(), W.cuda(), A[2].cuda(), B[2].cuda(), float(s[2]), 0.0, 1)
    assert float((S.float() - S1.float()).abs().max()) <= 2.0 ** -7 * float(S1.float().abs().max())
    assert float((Y.float() - Y1.float()).abs().max()) <= 2.0 ** -7 * float(Y1.float().abs().max())


def test_pool_past_32_bits():
    """The last adapter of a pool whose A and B each hold more than 2^31 elements."""
    P, r, K, N = 8200, 64, 4096, 4160
    g = gen(5)
    A, B = torch.zeros((P, r, K), dtype=BF16, device="cuda"), torch.zeros((P, N, r), dtype=BF16, device="cuda")
    a, b = normal(g, (2, r, K), K ** -0.5), normal(g, (2, N, r), 0.1)
    A[0], A[P - 1], B[0], B[P - 1] = a[0].cuda(), a[1].cuda(), b[0].cuda(), b[1].cuda()
    X, W = normal(g, (20, K)), normal(g, (N, K), K ** -0.5)
    ids = torch.tensor([0, P - 1] * 10, dtype=torch.int32)
    s = torch.ones(P)
    Y, S = binding.lora_requests_fwd(X.cuda(), W.cuda(), A, B, ids.cuda(), s.cuda())
    ref, bound, sref, sbound = requests(X, W, a, b, (ids > 0).int(), s[:2], None)
    within(S, sref, sbound, "S")
    within(Y, ref, bound, "Y")


def test_arguments():
    X, W, A, B, ids, s, _ = (None if t is None else t.cuda() for t in _case(8, 64, 64, 16, 2, "any", False, 1))
    with pytest.raises(AssertionError):
        binding.lora_requests_fwd(X, W, A, B, ids.long(), s)
    with pytest.raises(AssertionError):
        binding.lora_requests_fwd(X, W[:, :32], A, B, ids, s)
    with pytest.raises(AssertionError):
        binding.lora_requests_fwd(X.float(), W, A, B, ids, s)
    with pytest.raises(AssertionError):
        binding.lora_requests_fwd(X, W, A, B, ids[:4], s)
    Y, S = binding.lora_requests_fwd(X[:0], W, A, B, ids[:0], s)
    assert Y.shape == (0, 64) and S.shape == (0, 16)


@pytest.mark.parametrize("M,r", [(255, 64), (256, 64), (257, 64), (400, 64), (512, 32), (513, 32), (512, 16)])
def test_first_product_by_rows_or_tiles(M, r):
    """Both sides of the line between single rows and tiles of rows in the first product."""
    for ids in ("one", "chunks", "any"):
        _check(_case(M, 704, 192, r, 6, ids, True, M + r), (M, r, ids))


@pytest.mark.parametrize("M,r", [((1 << 21) - 1, 64), ((1 << 20) + 5, 16)])
def test_most_rows(M, r):
    """As many rows as the entry point takes, and a few more than one launch of the first product has."""
    print("requests", M, r, flush=True)
    K, N, P = 64, 64, 3
    W, A, B = (t.cuda() for t in _case(1, K, N, r, P, "one", False, 9)[1:4])
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    X = torch.randn((M, K), generator=g, device="cuda").to(BF16)
    ids = (torch.arange(M, device="cuda") // 37 % (P + 1) - 1).to(torch.int32)
    ids[-70:] = torch.arange(70, device="cuda", dtype=torch.int32) % P
    s = torch.tensor([0.5, -1.0, 2.0], device="cuda")
    Y, S = torch.full((M, N), 7.0, dtype=BF16, device="cuda"), torch.full((M, r), 7.0, dtype=BF16, device="cuda")
    binding.lora_requests_fwd(X, W, A, B, ids, s, Y=Y, S=S)
    for rows in torch.arange(M, device="cuda").split(1 << 19):
        x, of = X[rows].double(), ids[rows]
        y, sums = x @ W.double().t(), x.abs() @ W.double().abs().t() * (K * U32)
        t, tb = torch.zeros((rows.numel(), r), device="cuda", dtype=torch.float64), torch.zeros((rows.numel(), r), device="cuda", dtype=torch.float64)
        for i in range(P):
            at = of == i
            a, b, sg = A[i].double(), B[i].double(), float(s[i])
            t[at] = sg * (x[at] @ a.t())
            tb[at] = U16 * t[at].abs() + abs(sg) * (K + 2) * U32 * (x[at].abs() @ a.abs().t())
            y[at] += t[at] @ b.t()
            sums[at] += tb[at] @ b.abs().t() + (r + 1) * U32 * (t[at].abs() @ b.abs().t())
        assert bool(((S[rows].double() - t).abs() <= tb * (1 + U16)).all()), "S"
        assert bool(((Y[rows].double() - y).abs() <= sums * (1 + U16) + U16 * y.abs()).all()), "Y"
