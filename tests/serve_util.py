"""Plain 64-bit forms of the operators around served adapters, on the CPU, each with a bound on what an implementation may be off: 2^-8 of a value for
every rounding to bf16 (half a unit of its eight significant bits) and a share of the sum of magnitudes for sums in fp32."""
import math

import torch

U16, U32 = 2.0 ** -8, 2.0 ** -24
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def normal(g, shape, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g) * std + mean).to(BF16)


def within(got, ref, bound, label):
    """Every element within its bound; not-finite ones in the same places."""
    got, ref = got.detach().to("cpu", F64), ref.to(F64)
    assert got.shape == ref.shape, (label, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), (label, "not finite elsewhere", int((fine != torch.isfinite(got)).sum()))
    over = ((got - ref).abs() - bound.to(F64).expand_as(ref))[fine]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 0.0, (label, "over the bound by", worst, "max err", float((got - ref).abs()[fine].max()))


# ---- adapters of many requests ------------------------------------------------------------------------
def requests(X, W, A, B, ids, s, ranks):
    """Y, its bound, S and its bound."""
    P, N, r = B.shape
    M, K = X.shape
    X, W = X.to(F64), W.to(F64)
    Y, S = X @ W.t(), torch.zeros((M, r), dtype=F64)
    sums = X.abs() @ W.abs().t() * (K * U32)
    bound, s_bound = sums, torch.zeros((M, r), dtype=F64)
    for i in range(M):
        g = int(ids[i])
        if not 0 <= g < P:
            continue
        q = r if ranks is None else min(max(int(ranks[g]), 0), r)
        a, b, sg = A[g, :q].to(F64), B[g, :, :q].to(F64), abs(float(s[g]))
        S[i, :q] = float(s[g]) * (a @ X[i])
        s_bound[i, :q] = U16 * S[i, :q].abs() + sg * (K + 2) * U32 * (a.abs() @ X[i].abs())
        Y[i] += b @ S[i, :q]
        bound[i] += b.abs() @ s_bound[i, :q] + (r + 1) * U32 * (b.abs() @ S[i, :q].abs())
    return Y, bound * (1 + U16) + U16 * Y.abs(), S, s_bound * (1 + U16)


# ---- norm and rotation -----------------------------------------------------------------------------------
def _pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, c, s, interleaved):
    a, b = _pairs(2 * c.shape[-1], interleaved)
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def norm_rope(x, gamma, cos, sin, pos, eps, interleaved):
    """y [M,H,D] in 64 bits and its bound; differentiable in x and gamma."""
    known = ((pos >= 0) & (pos < cos.shape[0]))[:, None, None]
    at = pos.clamp(0, max(cos.shape[0] - 1, 0)).long()
    c, s = (t.to(F64)[at][:, None] if t.shape[0] else torch.zeros((pos.numel(), 1, t.shape[1]), dtype=F64) for t in (cos, sin))
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma
    y = torch.where(known, turn(n, c, s, interleaved), torch.zeros_like(n))
    mag = turn(n.detach().abs(), c.abs(), -s.abs(), interleaved)              # |a c| + |b s| in the first entry of a pair
    mag = torch.maximum(mag.abs(), turn(n.detach().abs(), c.abs(), s.abs(), interleaved).abs())
    a, b = _pairs(2 * c.shape[-1], interleaved)
    both = n.detach().abs()
    top = both[..., a] + both[..., b]
    mag[..., a], mag[..., b] = top, top
    return y, U16 * y.detach().abs() + (x.shape[-1] + 16) * U32 * mag


# ---- cache -----------------------------------------------------------------------------------------------------
def quantised(x):
    """e4m3 codes (uint8) and biased exponents of x [.., D] bf16, element by element from the definition."""
    codes = torch.zeros(x.shape, dtype=torch.uint8)
    exps = torch.zeros(x.shape[:-1], dtype=torch.uint8)
    flat, cf, ef = x.to(F64).reshape(-1, x.shape[-1]), codes.view(-1, x.shape[-1]), exps.view(-1)
    for row in range(flat.shape[0]):
        v = flat[row]
        top = max([abs(t) for t in v.tolist() if math.isfinite(t)], default=0.0)
        e = 0
        if top > 0:
            e = -117
            while top > 448.0 * 2.0 ** e:
                e += 1
        ef[row] = e + 127
        for j, t in enumerate(v.tolist()):
            sign = 0x80 if math.copysign(1.0, t) < 0 and not math.isnan(t) else 0
            if not math.isfinite(t):
                cf[row, j] = 0x7F
                continue
            a = abs(t) * 2.0 ** -e
            b = max(math.frexp(a)[1] - 1, -6) if a else -6
            m = a * 2.0 ** (3 - b)
            k = math.floor(m)
            k += m - k > 0.5 or (m - k == 0.5 and k % 2 == 1)
            cf[row, j] = sign | (k if b == -6 else k + ((b + 6) << 3))        # (a carry into the exponent comes out right)
    return codes, exps


def widened(codes, exps):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).to(F64), exps.to(torch.int32)[..., None] - 127)


# ---- attention --------------------------------------------------------------------------------------------------
def attention(q, k, v, n, kv, scale, window):
    """One sequence: q [n,H,D], k, v [kv,G,D] in 64 bits.  The result and its bound: each p is rounded to bf16 (2^-8 of it) and carries the error of its
    score in fp32, the result is rounded once."""
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    out, bound = torch.zeros((n, H, D), dtype=F64), torch.zeros((n, H, D), dtype=F64)
    pos = torch.arange(kv - n, kv)[:, None]
    key = torch.arange(kv)[None, :]
    seen = key <= pos
    if window:
        seen &= key > pos - window
    for h in range(H):
        g = h // (H // G)
        s = (q[:, h] @ k[:, g].t()) * scale
        size = (q[:, h].abs() @ torch.nan_to_num(k[:, g].abs(), 0.0, 0.0, 0.0).t()) * scale
        s = torch.where(seen, s, torch.full_like(s, -math.inf))
        top = s.amax(-1, keepdim=True) if kv else torch.zeros((n, 1), dtype=F64)
        p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(top), top)), torch.zeros_like(s))
        l = p.sum(-1, keepdim=True)
        p = torch.where(l > 0, p / l, p)
        vis = lambda w: torch.stack([(p[i][seen[i]][:, None] * w[seen[i]]).sum(0) for i in range(n)]) if n else out[:, h]
        out[:, h] = vis(v[:, g])
        off = float((torch.where(seen, size, torch.zeros_like(size))).max()) if n and kv else 0.0
        each = U16 + 4 * (D + 8) * U32 * max(1.0, off) + (kv + 8) * U32      # rounding of p; its score and exponential; the sums
        bound[:, h] = U16 * out[:, h].abs() + 1.01 * 2 * each * vis(v[:, g].abs())
    return out, bound
