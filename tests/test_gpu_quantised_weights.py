"""Weights in 4 bits: codes, exponents and what is read back, bit for bit."""
import pytest
import torch

from paper_2510_00206_amd import binding
from quant_util import quantised4, widened4
from serve_util import BF16, F64, gen, normal

pytestmark = pytest.mark.gpu


def _same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("N,K", [(64, 64), (128, 64), (64, 448), (320, 1088), (192, 4096), (1024, 192)])
def test_write_and_read(N, K):
    print("weights", N, K, flush=True)
    g = gen(N + K)
    W = (normal(g, (N, K)).float() * torch.exp2(torch.randint(-50, 50, (N, 1), generator=g).float())).to(BF16)
    W[0, :32] = 0
    W[1, :64] = -0.0
    W[2, 3], W[3, 33], W[4, 63] = float("inf"), float("nan"), -float("inf")
    codes, exps = torch.full((N, K // 2), 0x11, dtype=torch.uint8, device="cuda"), torch.full((N, K // 32), 0x11, dtype=torch.uint8, device="cuda")
    binding.lora_weights_write(W.cuda(), codes=codes, exps=exps)
    back = binding.lora_weights_read(codes, exps, W=torch.full((N, K), 7.0, dtype=BF16, device="cuda")).cpu()
    rc, re = quantised4(W)
    assert torch.equal(exps.cpu(), re)
    assert torch.equal(codes.cpu(), rc)
    ref = widened4(rc, re)
    nan = torch.isnan(ref)
    assert torch.equal(nan, torch.isnan(back)) and int(nan.sum()) == 96
    assert torch.equal(back.to(F64)[~nan], ref[~nan])


def test_every_code_and_exponent():
    """All pairs of codes under every exponent that a write gives, and NaN; zeros under the smaller ones."""
    exps = torch.arange(2, 253, dtype=torch.uint8).repeat_interleave(16)
    exps = torch.cat((exps, torch.full((5 * 16 + 64,), 255, dtype=torch.uint8)))
    exps = exps[:exps.numel() // 128 * 128]
    codes = torch.arange(exps.numel() * 16, dtype=torch.int64).remainder(256).to(torch.uint8)
    N, K = 64, exps.numel() * 32 // 64
    assert K % 64 == 0
    codes, exps = codes.view(N, K // 2), exps.view(N, K // 32)
    back = binding.lora_weights_read(codes.cuda(), exps.cuda()).cpu()
    ref = widened4(codes, exps)
    nan = torch.isnan(ref)
    assert torch.equal(nan, torch.isnan(back)) and torch.equal(back.to(F64)[~nan], ref[~nan])
    zero = binding.lora_weights_read(torch.zeros((64, 32), dtype=torch.uint8, device="cuda"), torch.zeros((64, 2), dtype=torch.uint8, device="cuda"))
    assert int((zero != 0).sum()) == 0


def test_borders():
    """Halfway between two codes goes to the even one, in every binade, and the power of two changes right past 6 times it."""
    rows = []
    for e in (-125, -120, -3, 0, 1, 60, 120):
        for top in (6.0, 6.03125, 3.0, 3.015625, 5.96875):
            row = torch.tensor([top, 0.25, 0.2490234375, 0.251953125, 0.75, 0.74609375, 1.25, 1.2578125, 1.75, 1.7421875, 2.5, 2.515625, 3.5, 3.484375, 5.0, 5.03125,
                                -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.0, -0.0, 4.0, 2.0, 1.0, 0.5, 1.5, 3.0, 0.0625], dtype=F64)
            rows.append(torch.where(row.abs() <= top, row, torch.full_like(row, top)) * 2.0 ** e)
    W = torch.stack(rows)[:35].repeat(64, 1)[:64 * 35].reshape(64, -1)
    W = W[:, :W.shape[1] // 64 * 64].contiguous().to(BF16)
    # ... and the least bf16 numbers there are
    W[5] = torch.arange(W.shape[1], dtype=torch.int16).view(BF16)
    W[6] = -W[5]
    codes, exps = binding.lora_weights_write(W.cuda())
    rc, re = quantised4(W)
    assert torch.equal(exps.cpu(), re) and torch.equal(codes.cpu(), rc)


def test_the_largest_values():
    """From 3.5 x 2^126 on they read as infinity."""
    W = torch.zeros((64, 64), dtype=BF16)
    W[0, 0], W[1, 0], W[2, 0] = 3.3895313892515355e38, 4.0 * 2.0 ** 126 * 0.99609375, 2.0 ** 127
    codes, exps = binding.lora_weights_write(W.cuda())
    back = binding.lora_weights_read(codes, exps).cpu().float()
    assert exps[:3, 0].tolist() == [253, 253, 252] and float(back[0, 0]) == float("inf") and float(back[2, 0]) == 2.0 ** 127


def test_the_training_layer_over_the_same_weights():
    """What is read feeds the training entry points: a forward and a backward over weights held in 4 bits, the gradients those of the 64-bit form."""
    M, N, K, r = 70, 192, 128, 16
    g = gen(4)
    X, A, B, dY = normal(g, (M, K)), normal(g, (r, K), K ** -0.5), normal(g, (N, r), 0.1), normal(g, (M, N))
    codes, exps = binding.lora_weights_write(normal(g, (N, K), K ** -0.5).cuda())
    W = binding.lora_weights_read(codes, exps)
    Y, S = binding.lora_fwd(X.cuda(), W, A.cuda(), B.cuda(), 2.0, 0.0, 1)
    dX, dA, dB = binding.lora_bwd(X.cuda(), W, A.cuda(), B.cuda(), S, dY.cuda(), 2.0, 0.0, 1)
    x, a, b = (t.to(F64).requires_grad_() for t in (X, A, B))
    y = x @ widened4(codes.cpu(), exps.cpu()).t() + 2.0 * (x @ a.t()) @ b.t()
    y.backward(dY.to(F64))
    served, _ = binding.lora_requests_quantised_fwd(X.cuda(), codes, exps, A[None].cuda(), B[None].cuda(), torch.zeros(M, dtype=torch.int32, device="cuda"),
                                                    torch.full((1,), 2.0, device="cuda"))
    # (three roundings to bf16 on the way to each: S or dS, and the result)
    for got, ref in ((Y, y.detach()), (served, y.detach()), (dX, x.grad), (dA, a.grad), (dB, b.grad)):
        assert float((got.cpu().to(F64) - ref).norm() / ref.norm()) <= 3 * 2.0 ** -8
