"""Norm and rotation of queries and keys against the 64-bit form, gradients against its derivative and against differences."""
import pytest
import torch

from paper_2510_00206_amd import binding
from serve_util import BF16, F32, F64, U16, U32, gen, norm_rope, normal, within

pytestmark = pytest.mark.gpu


def _inputs(M, H, G, D, rot, seed, positions=50, packed=True):
    g = gen(seed)
    qkv = normal(g, (M, (H + 2 * G) * D + (8 if packed else 0)))
    q, k = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + G) * D].unflatten(1, (G, D))
    gq, gk = normal(g, (D,), 0.3, 1.0), normal(g, (D,), 0.3, -0.5)
    ang = torch.rand((positions, rot // 2), generator=g) * 6.3
    pos = torch.randint(0, max(positions, 1), (M,), generator=g, dtype=torch.int32)
    return qkv, q, k, gq, gk, ang.cos(), ang.sin(), pos


CASES = [
    (1, 1, 1, 16, 16, False), (1, 32, 8, 128, 128, False), (3, 5, 2, 64, 32, True), (7, 8, 8, 80, 80, False), (2, 3, 1, 96, 48, False),
    (33, 4, 1, 256, 256, True), (50, 6, 2, 128, 64, False), (9, 7, 3, 208, 16, False), (64, 12, 4, 64, 64, False), (700, 3, 1, 128, 128, True),
    (1500, 9, 2, 48, 32, False), (4500, 2, 2, 128, 128, False),
]


@pytest.mark.parametrize("M,H,G,D,rot,inter", CASES)
def test_forward(M, H, G, D, rot, inter):
    print("norm_rope", M, H, G, D, rot, inter, flush=True)
    qkv, q, k, gq, gk, cos, sin, pos = _inputs(M, H, G, D, rot, M + D)
    if M > 2:
        pos[1], pos[2] = 50, -1                     # outside the tables: zeros
    dev = qkv.cuda()
    qd, kd = dev[:, :H * D].unflatten(1, (H, D)), dev[:, H * D:(H + G) * D].unflatten(1, (G, D))
    got = binding.lora_qk_norm_rope_fwd(qd, kd, *(t.cuda() for t in (gq, gk, cos, sin, pos)), eps=1e-5, interleaved=inter)
    for y, x, gamma, name in zip(got, (q, k), (gq, gk), "qk"):
        ref, bound = norm_rope(x.to(F64), gamma.to(F64), cos, sin, pos, 1e-5, inter)
        within(y, ref, bound, (name, M, H, G, D, rot, inter))
    # in place, as one part of the fused projection's output
    binding.lora_qk_norm_rope_fwd(qd, kd, *(t.cuda() for t in (gq, gk, cos, sin, pos)), eps=1e-5, interleaved=inter, q_out=qd, k_out=kd)
    assert torch.equal(qd, got[0]) and torch.equal(kd, got[1])
    assert torch.equal(dev[:, (H + G) * D:].cpu(), qkv[:, (H + G) * D:])


@pytest.mark.parametrize("M,H,G,D,rot,inter", CASES)
def test_backward(M, H, G, D, rot, inter):
    print("norm_rope backward", M, H, G, D, rot, inter, flush=True)
    qkv, q, k, gq, gk, cos, sin, pos = _inputs(M, H, G, D, rot, 1000 + M + D)
    if M > 2:
        pos[0], pos[2] = -5, 1 << 20
    g = gen(M)
    dy = normal(g, (M, H, D)), normal(g, (M, G, D))
    dev = qkv.cuda()
    qd, kd = dev[:, :H * D].unflatten(1, (H, D)), dev[:, H * D:(H + G) * D].unflatten(1, (G, D))
    args = (qd, kd, *(t.cuda() for t in (gq, gk, cos, sin, pos)), dy[0].cuda(), dy[1].cuda())
    got = binding.lora_qk_norm_rope_bwd(*args, eps=1e-5, interleaved=inter)
    sums = []
    for i, (x, gamma) in enumerate(((q, gq), (k, gk))):
        x, gamma = x.to(F64).clone().requires_grad_(), gamma.to(F64).clone().requires_grad_()
        y, _ = norm_rope(x, gamma, cos, sin, pos, 1e-5, inter)
        dx, dg = torch.autograd.grad(y, (x, gamma), dy[i].to(F64))
        # magnitudes that the sums run over: |R^T dy| <= |a| + |b| of a pair, times gamma / rms, and n times their mean
        with torch.no_grad():
            inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
            e = 2 * dy[i].to(F64).abs().amax(-1, keepdim=True)
            u = e * gamma.abs()
            mag = inv * (u + (x * inv).abs() * (u * (x * inv).abs()).mean(-1, keepdim=True))
            mag_g = (e * (x * inv).abs()).sum((0, 1))
        within(got[i], dx, U16 * dx.abs() + (D + 32) * U32 * mag, ("dx", i, M, H, D))
        # a chain of additions is at most rows x passes of a wave long, then lanes, waves and planes
        within(got[2 + i], dg, (D + 64 + 512) * U32 * mag_g, ("dgamma", i, M, H, D))
        sums.append(got[2 + i].clone())
    # the same bits again, and added to
    again = binding.lora_qk_norm_rope_bwd(*args, eps=1e-5, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    binding.lora_qk_norm_rope_bwd(*args, eps=1e-5, interleaved=inter, dgq=sums[0], dgk=sums[1], accumulate=True)
    assert torch.equal(sums[0], got[2] + got[2]) and torch.equal(sums[1], got[3] + got[3])


def test_gradient_against_differences():
    """The 64-bit form's central differences along a direction, against the gradients that the kernel returns: differences are exact to
    (step)^2, gradients to their rounding (2^-8 of each term of the product at most)."""
    M, H, G, D, rot = 6, 4, 2, 64, 32
    qkv, q, k, gq, gk, cos, sin, pos = _inputs(M, H, G, D, rot, 5)
    g = gen(9)
    dq_out, dk_out = normal(g, (M, H, D)), normal(g, (M, G, D))
    dq, dk, dgq, dgk = binding.lora_qk_norm_rope_bwd(*(t.cuda() for t in (q.contiguous(), k.contiguous(), gq, gk, cos, sin, pos, dq_out, dk_out)), eps=1e-5)
    for x, gamma, dy, dx, dg in ((q, gq, dq_out, dq, dgq), (k, gk, dk_out, dk, dgk)):
        x, gamma, dy = x.to(F64), gamma.to(F64), dy.to(F64)
        vx, vg = torch.randn(x.shape, generator=g, dtype=F64), torch.randn(gamma.shape, generator=g, dtype=F64)
        h = 1e-5
        loss = lambda t: float((norm_rope(x + t * vx, gamma + t * vg, cos, sin, pos, 1e-5, False)[0] * dy).sum())
        want = (loss(h) - loss(-h)) / (2 * h)
        terms = (dx.cpu().to(F64) * vx).abs().sum() + (dg.cpu().to(F64) * vg).abs().sum()
        got = float((dx.cpu().to(F64) * vx).sum() + (dg.cpu().to(F64) * vg).sum())
        assert abs(got - want) <= 2.0 ** -8 * float(terms) + 1e-6


def test_no_rows():
    _, q, k, gq, gk, cos, sin, pos = _inputs(4, 4, 2, 64, 64, 1)
    q, k, gq, gk, cos, sin, pos = (t.contiguous().cuda() for t in (q[:0], k[:0], gq, gk, cos, sin, pos[:0]))
    yq, yk = binding.lora_qk_norm_rope_fwd(q, k, gq, gk, cos, sin, pos)
    assert yq.shape == (0, 4, 64) and yk.shape == (0, 2, 64)
    dgq, dgk = torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda")
    binding.lora_qk_norm_rope_bwd(q, k, gq, gk, cos, sin, pos, q, k, dgq=dgq, dgk=dgk, accumulate=True)
    assert bool((dgq == 3).all()) and bool((dgk == 4).all())
    binding.lora_qk_norm_rope_bwd(q, k, gq, gk, cos, sin, pos, q, k, dgq=dgq, dgk=dgk)
    assert not dgq.any() and not dgk.any()


def test_empty_tables():
    """No positions at all: every row is outside them."""
    _, q, k, gq, gk, cos, sin, pos = _inputs(5, 4, 2, 64, 64, 1)
    y = binding.lora_qk_norm_rope_fwd(*(t.contiguous().cuda() for t in (q, k, gq, gk, cos[:0], sin[:0], pos)))
    assert not y[0].any() and not y[1].any()


def test_not_finite_stays_in_its_head():
    _, q, k, gq, gk, cos, sin, pos = _inputs(6, 4, 2, 64, 32, 3)
    q = q.clone()
    q[2, 1, 7], q[4, 3, 60] = float("nan"), float("inf")
    y, _ = binding.lora_qk_norm_rope_fwd(*(t.contiguous().cuda() for t in (q, k, gq, gk, cos, sin, pos)))
    bad = (~torch.isfinite(y)).any(-1).cpu()
    want = torch.zeros((6, 4), dtype=torch.bool)
    want[2, 1] = want[4, 3] = True
    assert torch.equal(bad, want)


def test_arguments():
    _, q, k, gq, gk, cos, sin, pos = (t.contiguous().cuda() for t in _inputs(4, 4, 2, 64, 64, 1))
    f = binding.lora_qk_norm_rope_fwd
    for bad in ((q.float(), k, gq, gk, cos, sin, pos), (q, k[:2], gq, gk, cos, sin, pos), (q, k, gq[:32], gk, cos, sin, pos),
                (q, k, gq, gk, cos.double(), sin, pos), (q, k, gq, gk, cos, sin, pos.long()), (q.transpose(1, 2).contiguous().transpose(1, 2), k, gq, gk, cos, sin, pos)):
        with pytest.raises(AssertionError):
            f(*bad)
    with pytest.raises(binding.LoraError):
        f(q, k, gq, gk, cos, sin, pos, eps=0.0)


@pytest.mark.parametrize("M,H,G,D,rot,inter", [(2100, 24, 8, 128, 128, False), (2100, 24, 8, 128, 64, True), (4200, 24, 8, 64, 64, False),
                                               (4200, 30, 2, 64, 32, True), (4200, 6, 2, 256, 256, False), (4200, 7, 1, 256, 128, True)])
def test_large_outputs(M, H, G, D, rot, inter):
    """Outputs of more than 16 MB, which go past the caches; backward with several parts of rows to a wave."""
    test_forward(M, H, G, D, rot, inter)
    test_backward(M, H, G, D, rot, inter)


@pytest.mark.parametrize("M,H,G,D,rot,inter", [(4, 3, 2, 64, 64, False), (40, 32, 8, 128, 128, False), (33, 4, 1, 256, 256, True), (50, 6, 2, 96, 48, False),
                                               (1500, 9, 2, 48, 32, True), (4500, 26, 2, 128, 128, False)])
def test_rows_outside_the_tables_add_nothing(M, H, G, D, rot, inter):
    """Rows of padding over memory that holds anything: zeros in dq and dk, and dgamma of the other rows alone (test_backward's bounds)."""
    print("rows outside", M, H, G, D, rot, inter, flush=True)
    _, q, k, gq, gk, cos, sin, pos = _inputs(M, H, G, D, rot, 77 + M)
    g = gen(M)
    xs, dys = [q.clone(), k.clone()], [normal(g, (M, H, D)), normal(g, (M, G, D))]
    out = torch.arange(M) % 3 == 1
    pos[out] = torch.tensor([-1, 50, 1 << 30, -(1 << 31)], dtype=torch.int32)[torch.arange(int(out.sum())) % 4]
    for t in xs + dys:
        t[out] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], dtype=BF16)[torch.randint(0, 4, t[out].shape, generator=g)]
    got = binding.lora_qk_norm_rope_bwd(*(t.cuda() for t in (*xs, gq, gk, cos, sin, pos, *dys)), eps=1e-5, interleaved=inter)
    for i, gamma in enumerate((gq, gk)):
        x, gamma, dy = xs[i][~out].to(F64).requires_grad_(), gamma.to(F64).requires_grad_(), dys[i][~out].to(F64)
        dx, dg = torch.autograd.grad(norm_rope(x, gamma, cos, sin, pos[~out], 1e-5, inter)[0], (x, gamma), dy)
        with torch.no_grad():
            inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
            e = 2 * dy.abs().amax(-1, keepdim=True)
            u = e * gamma.abs()
            mag = inv * (u + (x * inv).abs() * (u * (x * inv).abs()).mean(-1, keepdim=True))
            mag_g = (e * (x * inv).abs()).sum((0, 1))
        assert not got[i][out.cuda()].any()
        within(got[i][(~out).cuda()], dx, U16 * dx.abs() + (D + 32) * U32 * mag, ("dx", i))
        within(got[2 + i], dg, (D + 64 + 512) * U32 * mag_g, ("dgamma", i))


def test_most_rows():
    """As many rows as the entry points take; all hold one of 1000 rows, whose results the 64-bit form has."""
    M, some, D = (1 << 26) - 1, 1000, 16
    _, q, k, gq, gk, cos, sin, pos = (t.contiguous() for t in _inputs(some, 1, 1, D, 16, 8, packed=False))
    at = torch.arange(M, device="cuda") % some
    yq, yk = binding.lora_qk_norm_rope_fwd(*(t.cuda()[at] for t in (q, k)), gq.cuda(), gk.cuda(), cos.cuda(), sin.cuda(), pos.cuda()[at], eps=1e-5)
    for y, x, gamma in ((yq, q, gq), (yk, k, gk)):
        ref, bound = norm_rope(x.to(F64), gamma.to(F64), cos, sin, pos, 1e-5, False)
        within(y[:some], ref, bound, "first rows")
        for rows in y.split(some * 4000):
            n = rows.shape[0] // some * some
            assert bool((rows[:n].view(-1, some, D) == y[:some, 0]).all()) and torch.equal(rows[n:], y[:rows.shape[0] - n])


@pytest.mark.parametrize("inter", [False, True])
def test_entries_past_the_rotation_have_no_pair(inter):
    """An infinity in an entry that is not turned: the head's others are 0 (a norm over infinity), in its gradient dgamma of that entry alone is not finite."""
    M, H, G, D, rot = 6, 4, 2, 64, 32
    _, q, k, gq, gk, cos, sin, pos = _inputs(M, H, G, D, rot, 13)
    q, k = q.clone(), k.clone()
    q[2, 1, 40], k[4, 1, 63] = float("inf"), -float("inf")
    got = binding.lora_qk_norm_rope_fwd(*(t.contiguous().cuda() for t in (q, k, gq, gk, cos, sin, pos)), interleaved=inter)
    for y, x, gamma in zip(got, (q, k), (gq, gk)):
        ref = norm_rope(x.to(F64), gamma.to(F64), cos, sin, pos, 1e-6, inter)[0]
        assert torch.equal(torch.isfinite(y).cpu(), torch.isfinite(ref))
        hit = torch.isinf(x).any(-1)
        assert not y.cpu()[hit][torch.isfinite(ref)[hit]].any()
    _, q, k, *_ = _inputs(M, H, G, D, rot, 13)
    g = gen(2)
    dq_out, dk_out = normal(g, (M, H, D)), normal(g, (M, G, D))
    dq_out[1, 2, 41], dk_out[3, 0, 62] = float("inf"), -float("inf")
    _, _, dgq, dgk = binding.lora_qk_norm_rope_bwd(*(t.contiguous().cuda() for t in (q, k, gq, gk, cos, sin, pos, dq_out, dk_out)), interleaved=inter)
    for dg, entry in ((dgq, 41), (dgk, 62)):
        assert (~torch.isfinite(dg)).nonzero().flatten().tolist() == [entry]
