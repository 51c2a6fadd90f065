"""Workloads of the operators that serve adapters over 4 bits: the frozen weights and the paged cache of keys and values are held as e2m1 codes
(0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, two to a byte, the first in the low half) with a power of two for every 32 entries, a byte with its biased
exponent.  Inputs, the operators in plain torch, in 64 bits, and through the library's entry points (`paper_2510_00206_amd.binding`).

  weights     bf16 weights into that form and back
  layer       Y[i] = X[i] W^T + s_g (X[i] A_g^T) B_g^T, g = ids[i], W in that form: every row names its adapter, or none (-1)
  append      queries and keys: RMS norm over each head (or none), rotation by the row's position; queries out, keys and values into the slots of a paged
              cache (bf16, fp8 with a power of two for every token and head, or 4 bits)
  attend      attention of a few new tokens of each sequence over a 4-bit cache, causal, optionally over a window

A case is a dict of plain values, "op" first; what the others mean stands at _weights, _layer, _append and _attend.  Sizes are those of the
repository's layers (4096 = 32 heads of 128 with 8 key/value heads, 8192 = 64 heads; feed-forward 14336; ranks 16, 32, 64) and of
generic batches.  Values follow its input recipe: X ~ N(0,1), W ~ N(0,1/K), A ~ U(-K^-1/2, K^-1/2), B ~ N(0, 0.02^2), all bf16.
"""
import math

import torch

own = False

_BF16, _F32, _F64, _FP8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn


# ---- the cases -----------------------------------------------------------------------------------------
def _weights(name, do, N, K):
    """do: "read" (4 bits to bf16) | "write" (bf16 to 4 bits, and read: what a layer will see of them)."""
    return dict(op="weights", name=name, do=do, N=N, K=K)


def _layer(name, rows, K, N, r, pool, mixed=False):
    """rows: tokens of each request in the batch, "700,331,1*37" (37 requests of one token); pool: adapters held, 0: none and no ids; mixed: they
    use r or half or a quarter of it."""
    return dict(op="layer", name=name, rows=rows, K=K, N=N, r=r, pool=pool, mixed=mixed)


def _append(name, rows, heads, kv_heads, dim, rot, page, form, norm=True, interleaved=False, seqs=1):
    """rows: tokens, of `seqs` packed sequences; rot: rotated dimensions of a head, in pairs (i, i + rot/2) or, interleaved, (2i, 2i + 1);
    form of the cache: "bf16" | "fp8" | "fp4" (its rows are read back: the values that it stands for)."""
    return dict(op="append", name=name, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, page=page, form=form, norm=norm,
                interleaved=interleaved, seqs=seqs)


def _attend(name, seqs, new, kv_lo, kv_hi, heads, kv_heads, dim, page, window=0):
    """seqs sequences with `new` new tokens each (the last one fewer, if there are several) and kv_lo .. kv_hi tokens in the cache,
    the new ones among them."""
    return dict(op="attend", name=name, seqs=seqs, new=new, kv_lo=kv_lo, kv_hi=kv_hi, heads=heads, kv_heads=kv_heads, dim=dim, page=page, window=window)


def listed():
    return [
        # one token of one request on a small layer: launches and latency only
        _layer("layer_one", "1*1", 1024, 1024, 16, 4),
        # one decode step of 16 requests, fused query/key/value projection
        _layer("layer_decode", "1*16", 4096, 6144, 16, 12),
        # a large decode batch on the gate projection, adapters of different rank
        _layer("layer_decode_wide", "1*96", 4096, 14336, 64, 64, mixed=True),
        # a step that mixes chunks of three prompts with decoding requests, output projection
        _layer("layer_mixed", "700,331,1*37,980", 4096, 4096, 32, 12, mixed=True),
        # a small projection laid out for serving
        _weights("weights_write", "write", 1024, 4096),
        # a feed-forward projection widened for a training step on the same frozen weights
        _weights("weights_read", "read", 14336, 4096),
        # one decode step behind the fused projection
        _append("append_decode", 16, 32, 8, 128, 128, 16, "fp4", seqs=16),
        # a step with prompt chunks
        _append("append_chunks", 2085, 32, 8, 128, 128, 16, "fp4", seqs=3),
        # an unpadded batch, 64 heads, half of each head rotated in adjacent pairs, no norm, a cache that is not quantised
        _append("append_wide", 5003, 64, 8, 128, 64, 64, "bf16", norm=False, interleaved=True, seqs=3),
        # one decode step of 32 short and medium conversations
        _attend("attend_decode", 32, 1, 200, 4000, 32, 8, 128, 16),
        # a decode step of four long documents
        _attend("attend_decode_long", 4, 1, 33000, 131072, 32, 8, 128, 64),
        # two prompts' next chunks over what of them is in the cache
        _attend("attend_chunks", 2, 1021, 5003, 16000, 32, 8, 128, 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


def draw(rng):
    caps = {}
    for c in listed():
        caps[c["op"]] = max(caps.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choice(("layer", "layer", "weights", "append", "attend", "attend"))
        if op == "layer":
            K, N = (max(64, _log_int(rng, 256, 14336) // 64 * 64) for _ in range(2))
            r, pool = rng.choice((16, 32, 64)), rng.choice((0, _log_int(rng, 1, 128), _log_int(rng, 1, 128)))
            rows = "1*%d" % _log_int(rng, 1, 256)
            if rng.random() < 0.4:
                rows = ",".join([str(_log_int(rng, 2, 1024)) for _ in range(rng.randint(1, 4))] + [rows])
            case = _layer("", rows, K, N, r if pool else 0, pool, mixed=pool > 0 and rng.random() < 0.5)
            fits = sum(_rows(case)) * r * max(K, N) <= 2 ** 31 and pool * r * max(K, N) <= 2 ** 29
        elif op == "weights":
            case = _weights("", rng.choice(("read", "write")), max(64, _log_int(rng, 256, 14336) // 64 * 64), max(64, _log_int(rng, 256, 14336) // 64 * 64))
            fits = True
        elif op == "append":
            kv = rng.choice((1, 2, 4, 8))
            form = rng.choice(("bf16", "fp8", "fp4", "fp4"))
            dim = rng.choice((64, 96, 128, 128, 256) if form == "fp4" else (64, 80, 128, 128, 256))
            rows = _log_int(rng, 1, 6000)
            case = _append("", rows, kv * rng.choice((1, 2, 3, 4, 8)), kv, dim, rng.choice((dim, dim, 16 * max(1, dim // 32))),
                           rng.choice((16, 32, 64)), form, rng.random() < 0.7, rng.random() < 0.3, min(rows, rng.choice((1, 2, 5))))
            fits = True
        else:
            kv, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128))
            seqs = _log_int(rng, 1, 64)
            new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 2048)
            hi = _log_int(rng, max(new, 32), 65536)
            lo = max(new, int(hi * rng.uniform(0.02, 1.0)))
            case = _attend("", seqs, new, lo, hi, kv * rng.choice((1, 3, 4, 7, 8)), kv, dim, rng.choice((16, 32, 64)),
                           rng.choice((0, 0, 0, _log_int(rng, 16, 8192))))
            fits = seqs * case["heads"] * new * hi <= 1 << 30 and seqs * hi * kv * dim <= 1 << 29
        if fits and _cost(case) <= caps[op]:
            del case["name"]
            return case


# ---- inputs ----------------------------------------------------------------------------------------------
def _rows(case):
    out = []
    for part in case["rows"].split(","):
        n, _, times = part.partition("*")
        out += [int(n)] * int(times or 1)
    return out


def _new_tokens(case):
    n = [case["new"]] * case["seqs"]
    if len(n) > 1:
        n[-1] = max(1, n[-1] * 2 // 3)
    return n


def _kv_lens(case):
    """Spread over kv_lo .. kv_hi in an order that is not sorted."""
    b, lo, hi = case["seqs"], case["kv_lo"], case["kv_hi"]
    return [lo + (i * 37 % b) * (hi - lo) // max(1, b - 1) if b > 1 else hi for i in range(b)]


class _State:
    pass


class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) % (1 << 63))

    def normal(self, shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=self.g, device="cuda", dtype=_F32) * std + mean).to(_BF16)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=_F32)

    def ints(self, lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda")

    def permutation(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _exponents(top, largest, least):
    """The smallest e (at least `least`; 0 for 0) with top <= largest * 2^e, largest = m 2^n with 0.5 <= m < 1."""
    m, n = math.frexp(largest)
    f, e = torch.frexp(top)
    e = torch.where(f > m, e - n + 1, e - n)
    return torch.where(top == 0, torch.zeros_like(e), e).clamp(min=least)


def _to_fp8(x):
    """e4m3 values and the biased exponents of a power of two over the last dimension of x (32 or 64 bits)."""
    e = _exponents(x.abs().amax(dim=-1), 448.0, -117)
    return _odd(torch.ldexp(x, -e[..., None])).to(_FP8), (e + 127).to(torch.uint8)


def _odd(x):
    """x in 32 bits, what that leaves of 64 kept in the last one, so that another rounding is as if from x."""
    y = x.to(_F32)
    if x.dtype is _F32:
        return y
    bits = y.view(torch.int32)
    gone = x.abs() - y.abs().to(_F64)
    return torch.where((gone != 0) & (bits & 1 == 0), torch.where(gone > 0, bits + 1, bits - 1), bits).view(_F32)


def _to_fp4(x):
    """Codes [.., n/2] and biased exponents [.., n/32] of x [.., n] (32 or 64 bits)."""
    x = x.unflatten(-1, (-1, 32))
    e = _exponents(x.abs().amax(dim=-1), 6.0, -125)
    a = torch.ldexp(x, -e[..., None])
    sign = torch.signbit(a)
    a = a.abs()
    code = (a > 0.25).to(torch.uint8)
    for above in (0.75 <= a, a > 1.25, 1.75 <= a, a > 2.5, 3.5 <= a, a > 5.0):       # halfway goes to the even code
        code += above
    code = (code + 8 * sign.to(torch.uint8)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _from_fp4(codes, exps):
    """Their values [.., n] in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=_F32, device=codes.device)
    x = table[torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int32)]
    return torch.ldexp(x.unflatten(-1, (-1, 32)), exps.to(torch.int32)[..., None] - 127).flatten(-2)


def prepare(case, seed):
    st, rnd = _State(), _Random(seed)
    st.case = case
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    if case["op"] == "weights":
        N, K = case["N"], case["K"]
        W = rnd.normal((N, K), K ** -0.5)
        if case["do"] == "read":
            st.codes, st.exps = _to_fp4(W.to(_F32))
        else:
            st.W, st.codes, st.exps = W, new((N, K // 2), torch.uint8), new((N, K // 32), torch.uint8)
        st.out = new((N, K), _BF16)
    elif case["op"] == "layer":
        K, N, r, P = case["K"], case["N"], case["r"], case["pool"]
        lens = _rows(case)
        M = sum(lens)
        st.X = rnd.normal((M, K))
        st.codes, st.exps = _to_fp4(rnd.normal((N, K), K ** -0.5).to(_F32))
        st.A = st.B = st.ids = st.s = st.ranks = st.S = None
        if P:
            st.A = ((rnd.uniform((P, r, K)) * 2 - 1) * K ** -0.5).to(_BF16)
            st.B = rnd.normal((P, N, r), 0.02)
            st.s = torch.tensor([0.5, 1.0, 2.0], device="cuda")[rnd.ints(0, 3, (P,))]
            st.ranks = torch.tensor([r, r // 2, r // 4], device="cuda", dtype=torch.int32)[rnd.ints(0, 3, (P,))] if case["mixed"] else None
            of = (P * rnd.uniform((len(lens),)) ** 2).to(torch.int32).clamp(max=P - 1)      # some tenants ask more often than others
            of = torch.where(rnd.uniform((len(lens),)) < 0.1, torch.full_like(of, -1), of)  # ... and some for the base model
            st.ids = torch.repeat_interleave(of, torch.tensor(lens, device="cuda"))
            st.S = new((M, r), _BF16)
        st.Y = new((M, N), _BF16)
    elif case["op"] == "append":
        M, H, G, D, rot, page = (case[k] for k in ("rows", "heads", "kv_heads", "dim", "rot", "page"))
        spread = torch.exp(rnd.uniform((M, G, 1)) * 4 - 2)               # tokens and heads of the values differ in magnitude
        st.qkv = torch.cat((rnd.normal((M, (H + G) * D)), (rnd.normal((M, G, D)) * spread).to(_BF16).view(M, G * D)), dim=1)
        st.q, st.k, st.v = (st.qkv[:, a * D:b * D].view(M, b - a, D) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        st.gq = st.gk = None
        if case["norm"]:
            st.gq, st.gk = rnd.normal((D,), 0.1, 1.0), rnd.normal((D,), 0.1, 1.0)
        per = -(-M // case["seqs"])
        if M <= 4 * case["seqs"]:                                        # decoding: anywhere in a context
            per, st.pos = 8192, rnd.ints(0, 8192, (M,)).to(torch.int32)
        else:                                                            # packed sequences
            st.pos = (torch.arange(M, device="cuda") % per).to(torch.int32)
        ang = torch.arange(per, device="cuda", dtype=_F64)[:, None] * 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=_F64) / (rot // 2))
        st.cos, st.sin, st.eps = ang.cos().to(_F32), ang.sin().to(_F32), 1e-6
        pages = -(-M // page) + 8
        at = rnd.permutation(pages)[:, None] * page + torch.arange(page, device="cuda")
        st.slots = at.reshape(-1)[:M].contiguous()
        width, dtype = {"bf16": (D, _BF16), "fp8": (D, _FP8), "fp4": (D // 2, torch.uint8)}[case["form"]]
        exps = {"bf16": None, "fp8": (pages, G, page), "fp4": (pages, G, page, D // 32)}[case["form"]]
        st.pages = tuple(torch.zeros((pages, G, page, width), dtype=dtype, device="cuda") for _ in range(2)) + \
            tuple(None if exps is None else torch.zeros(exps, dtype=torch.uint8, device="cuda") for _ in range(2))
        st.q_out, st.k_out, st.v_out = new((M, H, D), _BF16), new((M, G, D), _BF16), new((M, G, D), _BF16)
    else:
        H, G, D, page = (case[k] for k in ("heads", "kv_heads", "dim", "page"))
        n, kv = _new_tokens(case), _kv_lens(case)
        used = [-(-v // page) for v in kv]
        pages = sum(used) + 4
        (k, ke), (v, ve) = (_to_fp4(rnd.normal((pages, G, page, D), std).to(_F32)) for std in (0.6, 1.0))
        st.pages = k, v, ke, ve
        order = rnd.permutation(pages)[:sum(used)].to(torch.int32)
        used = torch.tensor(used, device="cuda")
        st.table = torch.zeros((len(n), int(used.max())), dtype=torch.int32, device="cuda")
        st.table[torch.arange(st.table.shape[1], device="cuda")[None, :] < used[:, None]] = order
        st.n, st.max_new, st.max_kv = n, max(n), max(kv)
        st.offsets = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device="cuda")
        st.kv_lens = torch.tensor(kv, dtype=torch.int32, device="cuda")
        st.q, st.out = rnd.normal((sum(n), H, D), 2.0), new((sum(n), H, D), _BF16)
        st.ws = None
    return st


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    return {"weights": _run_weights, "layer": _run_layer, "append": _run_append, "attend": _run_attend}[st.case["op"]](st)


def _run_weights(st):
    if own:
        from paper_2510_00206_amd import binding
        if st.case["do"] == "write":
            binding.lora_weights_write(st.W, codes=st.codes, exps=st.exps)
        return binding.lora_weights_read(st.codes, st.exps, W=st.out)
    if st.case["do"] == "write":
        st.codes, st.exps = _to_fp4(st.W.to(_F32))
    return _from_fp4(st.codes, st.exps).to(_BF16)


def _run_layer(st):
    if own:
        from paper_2510_00206_amd import binding
        return binding.lora_requests_quantised_fwd(st.X, st.codes, st.exps, st.A, st.B, st.ids, st.s, ranks=st.ranks, Y=st.Y, S=st.S)[0]
    X = st.X.to(_F32)
    Y = X @ _from_fp4(st.codes, st.exps).t()
    if st.ids is None:
        return Y.to(_BF16)
    g = st.ids.clamp(min=0)
    S = torch.bmm(st.A[g].to(_F32), X[:, :, None])[:, :, 0] * st.s[g][:, None]
    used = (st.ids >= 0)[:, None].expand_as(S)
    if st.ranks is not None:
        used = used & (torch.arange(S.shape[1], device=S.device)[None, :] < st.ranks[g][:, None])
    S = torch.where(used, S, torch.zeros_like(S))
    return (Y + torch.bmm(st.B[g].to(_F32), S[:, :, None])[:, :, 0]).to(_BF16)


def _rotate(x, cos, sin, interleaved):
    """The pairs of the first 2 * cos.shape[-1] entries turned by their angles; the others as they are."""
    half = cos.shape[-1]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        head = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((head, rest), dim=-1)


def _run_append(st):
    case = st.case
    k, v, ke, ve = st.pages
    if own:
        from paper_2510_00206_amd import binding
        cache = binding.KVCache(k, v, ke, ve)
        binding.lora_kv_cache_append(cache, st.q, st.k, st.v, st.cos, st.sin, st.pos, st.slots, gq=st.gq, gk=st.gk, eps=st.eps,
                                     interleaved=case["interleaved"], q_out=st.q_out)
        if case["form"] == "fp4":
            return (st.q_out, *binding.lora_kv_cache_read(cache, st.slots, k=st.k_out, v=st.v_out))
        return (st.q_out, k, v) if ke is None else (st.q_out, k, v, ke, ve)
    turned = []
    for x, gamma, t in ((st.q, st.gq, _F32), (st.k, st.gk, _F64)):       # (keys are next to the borders of the quantiser's steps)
        x = x.to(t)
        if gamma is not None:
            x = x * (1.0 / torch.sqrt(torch.mean(x * x, dim=-1, keepdim=True) + st.eps)) * gamma.to(t)
        turned.append(_rotate(x, st.cos[st.pos.long()][:, None].to(t), st.sin[st.pos.long()][:, None].to(t), case["interleaved"]))
    q_out, page = turned[0].to(_BF16), k.shape[2]
    at = (st.slots // page, slice(None), st.slots % page)
    for x, e, new in ((k, ke, turned[1]), (v, ve, st.v.to(_F32))):
        if case["form"] == "bf16":
            x[at] = new.to(_BF16)
        else:
            codes, exps = (_to_fp8 if case["form"] == "fp8" else _to_fp4)(new)
            x.view(torch.uint8)[at] = codes.view(torch.uint8)
            e[at] = exps
    if case["form"] == "fp4":
        return q_out, _from_fp4(k[at], ke[at]).to(_BF16), _from_fp4(v[at], ve[at]).to(_BF16)
    return (q_out, k, v) if ke is None else (q_out, k, v, ke, ve)


def _run_attend(st):
    case = st.case
    k, v, ke, ve = st.pages
    if own:
        from paper_2510_00206_amd import binding
        cache = binding.KVCache(k, v, ke, ve)
        if st.ws is None:                                            # kept from step to step, as a serving program keeps it
            st.ws = binding.alloc_paged_attn_workspace(cache, st.q.shape[0], st.q.shape[1], st.table.shape[0], st.max_new, st.max_kv, case["window"])
        return binding.lora_paged_attn_fwd(st.q, cache, st.table, st.offsets, st.kv_lens, st.max_new, st.max_kv, window=case["window"],
                                           out=st.out, workspace=st.ws)
    H, G, D, page = (case[x] for x in ("heads", "kv_heads", "dim", "page"))
    B, n, L = st.table.shape[0], st.max_new, st.table.shape[1] * page
    # every sequence padded to the longest: queries [B, G, H/G * n, D], keys and values [B, G, L, D]
    new = st.offsets[1:] - st.offsets[:-1]
    step = torch.arange(n, device=k.device)
    at = (st.offsets[:-1, None] + step[None, :]).clamp(max=st.q.shape[0] - 1).long()
    q = st.q[at].to(_F32).view(B, n, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * n, D)
    K, V = (_from_fp4(x[st.table.long()], e[st.table.long()]).transpose(1, 2).reshape(B, G, L, D) for x, e in ((k, ke), (v, ve)))
    s = torch.matmul(q, K.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, G, H // G, n, L)
    pos = (st.kv_lens - new)[:, None] + step[None, :]                # of each query, [B, n]
    key = torch.arange(L, device=k.device)
    hidden = key[None, None, :] > pos[:, :, None]
    if case["window"]:
        hidden = hidden | (key[None, None, :] <= pos[:, :, None] - case["window"])
    s = s.masked_fill_(hidden[:, None, None], -math.inf)
    s = s.sub_(s.amax(dim=-1, keepdim=True)).exp_()
    s = s.div_(s.sum(dim=-1, keepdim=True))
    o = torch.matmul(s.view(B, G, H // G * n, L), V).view(B, G, H // G, n, D).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    return o[step[None, :] < new[:, None]].to(_BF16)


# ---- what a pass cannot do without ------------------------------------------------------------------------------
_BITS4 = 0.5 + 1.0 / 32                                               # bytes of an entry


def work(case):
    if case["op"] == "weights":
        n = case["N"] * case["K"]
        # written: read once in bf16, held; both: read from there, once more in bf16
        return {"bytes": n * (_BITS4 + 2 if case["do"] == "read" else 2 + 2 * _BITS4 + 2), "flops": n * (1 if case["do"] == "read" else 4)}
    if case["op"] == "layer":
        M, K, N, r, P = sum(_rows(case)), case["K"], case["N"], case["r"], case["pool"]
        # adapters in use: at most one to a request, and of a pool drawn with the square of a uniform number about so many
        n = len(_rows(case))
        used = sum(1.0 - (1.0 - (math.sqrt((g + 1) / P) - math.sqrt(g / P))) ** (0.9 * n) for g in range(P))
        mean_r = r * 7 / 12 if case["mixed"] else r
        return {"bytes": 2 * M * (K + N) + N * K * _BITS4 + 2 * used * mean_r * (K + N), "flops": 2 * M * K * N + 2 * 0.9 * M * mean_r * (K + N)}
    if case["op"] == "append":
        M, H, G, D, rot = case["rows"], case["heads"], case["kv_heads"], case["dim"], case["rot"]
        held = {"bf16": 2.0, "fp8": 1 + 1 / D, "fp4": _BITS4}[case["form"]]
        back = 2 * M * G * D * (held + 2) if case["form"] == "fp4" else 0      # (read back)
        return {"bytes": 2 * M * D * (H + 2 * G) + 2 * M * H * D + 2 * M * G * D * held + back + 4 * min(M, -(-M // case["seqs"])) * rot + 12 * M,
                "flops": (6 if case["norm"] else 3) * M * (H + G) * D + 4 * M * G * D}
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    w = case["window"] or 1 << 40
    pairs = keys = 0
    for n, kv in zip(_new_tokens(case), _kv_lens(case)):
        pairs += sum(min(w, kv - n + i + 1) for i in range(n))
        keys += min(kv, w + n - 1)
    return {"bytes": 2 * 2 * sum(_new_tokens(case)) * H * D + 2 * keys * G * D * _BITS4, "flops": 4 * pairs * H * D}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------
def _e2m1(codes, exps):
    """Values of 4-bit codes from their fields: sign, two exponent bits, one fraction bit."""
    c = torch.stack((codes.to(torch.int32) % 16, codes.to(torch.int32) // 16), dim=-1).flatten(-2)
    e, f = c // 2 % 4, (c % 2).to(_F64)
    x = torch.where(e > 0, (1 + f / 2) * torch.exp2(e.to(_F64) - 1), f / 2) * (1 - 2 * (c // 8)).to(_F64)
    return x * torch.exp2(exps.to(_F64) - 127).repeat_interleave(32, dim=-1)


def _rounded(x, top, largest, fraction, least_step, least):
    """x over its power of two, rounded to the nearest with `fraction` bits behind the first one (ties to even), and back."""
    e = torch.where(top > 0, torch.ceil(torch.log2(top / largest)), torch.zeros_like(top)).clamp(min=least)
    a = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=1e-300))) - fraction).clamp(min=least_step)
    a = torch.round(a / step) * step
    return a, torch.exp2(e)


def _held4(x):
    x = x.unflatten(-1, (-1, 32))
    a, by = _rounded(x, x.abs().amax(-1, keepdim=True), 6.0, 1, 0.5, -125)
    return (a * by).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "weights":
        return _held4(st.W.to(_F64)) if case["do"] == "write" else _e2m1(st.codes, st.exps)
    if case["op"] == "layer":
        X = st.X.to(_F64)
        Y = X @ _e2m1(st.codes, st.exps).t()
        for g in [] if st.ids is None else torch.unique(st.ids).tolist():
            if g < 0:
                continue
            q = case["r"] if st.ranks is None else int(st.ranks[g])
            at = (st.ids == g).nonzero()[:, 0]
            Y[at] += float(st.s[g]) * ((X[at] @ st.A[g, :q].to(_F64).t()) @ st.B[g, :, :q].to(_F64).t())
        return Y
    if case["op"] == "append":
        half, inter = case["rot"] // 2, case["interleaved"]
        i = torch.arange(half, device="cuda")
        first, second = (2 * i, 2 * i + 1) if inter else (i, i + half)
        turn = torch.complex(st.cos.to(_F64), st.sin.to(_F64))[st.pos.long()][:, None, :]
        ys = []
        for x, gamma in ((st.q, st.gq), (st.k, st.gk)):
            y = x.to(_F64)
            if gamma is not None:
                y = y / (y.square().sum(-1, keepdim=True) / case["dim"] + st.eps).sqrt() * gamma.to(_F64)
            z = torch.complex(y[..., first], y[..., second]) * turn
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            ys.append(y)
        if case["form"] == "fp4":
            return ys[0], _held4(ys[1]), _held4(st.v.to(_F64))
        page = st.pages[0].shape[2]
        out = [x.to(_F32).to(_F64) for x in st.pages[:2]]
        for x, new in zip(out, (ys[1], st.v.to(_F64))):
            if case["form"] == "fp8":
                new = _rounded(new, new.abs().amax(-1, keepdim=True), 448.0, 3, 2.0 ** -9, -117)[0]
            x[st.slots // page, :, st.slots % page] = new
        return (ys[0], *out) if case["form"] == "bf16" else (ys[0], *out, None, None)
    if sum(_new_tokens(case)) * case["heads"] * case["kv_hi"] > 1 << 31:
        return None
    k, v, ke, ve = st.pages
    page, G, D = k.shape[2], case["kv_heads"], case["dim"]
    out = torch.empty(st.q.shape, dtype=_F64, device="cuda")
    for b, (n, kv) in enumerate(zip(_new_tokens(case), _kv_lens(case))):
        pg = st.table[b, :-(-kv // page)].long()
        row = int(st.offsets[b])
        for g in range(G):
            Kg, Vg = (_e2m1(x[pg, g], e[pg, g]).reshape(-1, D)[:kv] for x, e in ((k, ke), (v, ve)))
            i = torch.arange(kv - n, kv, device="cuda")[:, None] - torch.arange(kv, device="cuda")[None, :]
            seen = (i >= 0) & (i < (case["window"] or 1 << 40))
            for h in range(g * (case["heads"] // G), (g + 1) * (case["heads"] // G)):
                s = (st.q[row:row + n, h].to(_F64) @ Kg.t()) / math.sqrt(D)
                out[row:row + n, h] = torch.softmax(torch.where(seen, s, torch.full_like(s, -math.inf)), dim=-1) @ Vg
    return out
