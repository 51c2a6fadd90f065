"""Workloads of the operators that serve adapters after they were trained, and of the one that stands behind the query
and key projections in training: inputs, the operators in plain torch, in 64 bits, and through the library's entry points
(`paper_2510_00206_amd.binding`).

  requests    Y[i] = X[i] W^T + s_g (X[i] A_g^T) B_g^T, g = ids[i]: every row names its adapter, or none (-1)
  norm_rope   queries and keys: RMS norm over each head, then the rotation by the row's position; forward and backward
  cache       keys and values into the slots of a paged cache (bf16, or fp8 with a power of two for every token and head) and back
  attend      attention of a few new tokens of each sequence over that cache, causal, optionally over a window

A case is a dict of plain values, "op" first; what the others mean stands at _requests, _norm_rope, _cache and _attend.  Sizes
are those of the repository's layers (4096 = 32 heads of 128 with 8 key/value heads, 8192 = 64 heads; feed-forward 14336; ranks
16, 32, 64) and of generic batches.  Values follow its input recipe: X ~ N(0,1), W ~ N(0,1/K), A ~ U(-K^-1/2, K^-1/2),
B ~ N(0, 0.02^2), all bf16.
"""
import math

import torch

own = False

_BF16, _F32, _F64 = torch.bfloat16, torch.float32, torch.float64


# ---- the cases -----------------------------------------------------------------------------------------
def _requests(name, rows, K, N, r, pool, mixed=False):
    """rows: tokens of each request in the batch, "700,331,1*37" (37 requests of one token); pool: adapters held; mixed: they use r
    or half or a quarter of it."""
    return dict(op="requests", name=name, rows=rows, K=K, N=N, r=r, pool=pool, mixed=mixed)


def _norm_rope(name, do, rows, heads, kv_heads, dim, rot, interleaved=False, seqs=1):
    """do: "fwd" | "bwd"; rows: tokens, of `seqs` packed sequences; rot: rotated dimensions of a head, in pairs (i, i + rot/2) or,
    interleaved, (2i, 2i + 1)."""
    return dict(op="norm_rope", name=name, do=do, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, interleaved=interleaved, seqs=seqs)


def _cache(name, do, rows, kv_heads, dim, page, fp8):
    """do: "write" | "read"; rows: tokens; page: tokens of a page."""
    return dict(op="cache", name=name, do=do, rows=rows, kv_heads=kv_heads, dim=dim, page=page, fp8=fp8)


def _attend(name, seqs, new, kv_lo, kv_hi, heads, kv_heads, dim, page, fp8, window=0):
    """seqs sequences with `new` new tokens each (the last one fewer, if there are several) and kv_lo .. kv_hi tokens in the cache,
    the new ones among them."""
    return dict(op="attend", name=name, seqs=seqs, new=new, kv_lo=kv_lo, kv_hi=kv_hi, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                fp8=fp8, window=window)


def listed():
    return [
        # three requests, one token each, on a small layer: launches and latency only
        _requests("requests_few", "1*3", 1024, 1024, 16, 4),
        # one decode step of 64 requests with their tenants' adapters, fused query/key/value projection
        _requests("requests_decode", "1*64", 4096, 6144, 16, 48),
        # a large decode batch on the gate projection, a full pool of adapters of different rank
        _requests("requests_decode_wide", "1*200", 4096, 14336, 64, 256, mixed=True),
        # a step that mixes chunks of three prompts with decoding requests, output projection
        _requests("requests_mixed", "700,331,1*37,980", 4096, 4096, 32, 12, mixed=True),
        # one decode step behind the fused projection
        _norm_rope("norm_rope_decode", "fwd", 16, 32, 8, 128, 128, seqs=16),
        # a training batch of four sequences
        _norm_rope("norm_rope_train", "fwd", 8192, 32, 8, 128, 128, seqs=4),
        # its backward: an unpadded batch, 64 heads, half of each head rotated in adjacent pairs
        _norm_rope("norm_rope_train_bwd", "bwd", 5003, 64, 8, 128, 64, interleaved=True, seqs=3),
        # the keys and values of a step with prompt chunks, quantised into pages of 16
        _cache("cache_write_chunks", "write", 2085, 8, 128, 16, True),
        # a shared prefix read back
        _cache("cache_read_prefix", "read", 29999, 8, 128, 64, True),
        # one decode step of 32 short and medium conversations over a quantised cache
        _attend("attend_decode", 32, 1, 200, 4000, 32, 8, 128, 16, True),
        # a decode step of four long documents
        _attend("attend_decode_long", 4, 1, 33000, 131072, 32, 8, 128, 64, False),
        # two prompts' next chunks over what of them is in the cache
        _attend("attend_chunks", 2, 1021, 5003, 16000, 32, 8, 128, 32, False),
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
        op = rng.choice(("requests", "requests", "norm_rope", "cache", "attend", "attend"))
        if op == "requests":
            K, N = (max(64, _log_int(rng, 256, 14336) // 64 * 64) for _ in range(2))
            r, pool = rng.choice((16, 32, 64)), _log_int(rng, 1, 256)
            rows = "1*%d" % _log_int(rng, 1, 384)
            if rng.random() < 0.5:
                rows = ",".join([str(_log_int(rng, 2, 1024)) for _ in range(rng.randint(1, 4))] + [rows])
            case = _requests("", rows, K, N, r, pool, mixed=rng.random() < 0.5)
            fits = sum(_rows(case)) * r * max(K, N) <= 2 ** 31 and pool * r * max(K, N) <= 2 ** 29
        elif op == "norm_rope":
            kv = rng.choice((1, 2, 4, 8))
            dim = rng.choice((64, 80, 96, 128, 128, 256))
            rows = _log_int(rng, 1, 16384)
            case = _norm_rope("", rng.choice(("fwd", "bwd")), rows, kv * rng.choice((1, 2, 3, 4, 8)), kv, dim,
                              rng.choice((dim, dim, 16 * max(1, dim // 32))), rng.random() < 0.3, min(rows, rng.choice((1, 2, 5))))
            fits = True
        elif op == "cache":
            case = _cache("", rng.choice(("write", "read")), _log_int(rng, 1, 32768), rng.choice((1, 2, 4, 8)), rng.choice((64, 128)),
                          rng.choice((16, 32, 64)), rng.random() < 0.7)
            fits = True
        else:
            kv, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128))
            seqs = _log_int(rng, 1, 64)
            new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 2048)
            hi = _log_int(rng, max(new, 32), 65536)
            lo = max(new, int(hi * rng.uniform(0.02, 1.0)))
            case = _attend("", seqs, new, lo, hi, kv * rng.choice((1, 3, 4, 7, 8)), kv, dim, rng.choice((16, 32, 64)), rng.random() < 0.5,
                           rng.choice((0, 0, 0, _log_int(rng, 16, 8192))))
            fits = seqs * case["heads"] * new * hi <= 1 << 30 and seqs * hi * kv * dim <= 1 << 29
        fits = fits and 3072 not in (case.get("K"), case.get("N"), case.get("rows"), case.get("heads", 0) * case.get("dim", 0))   # (none of the layers here)
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


def _quantised(x):
    """fp8 (e4m3) values and the biased exponents of their scales, over the last dimension of x: the scale is the smallest power of
    two (2^-117 at least) that keeps the largest magnitude within 448."""
    top = x.to(_F32).abs().amax(dim=-1)
    m, e = torch.frexp(top)                                          # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(top == 0, torch.zeros_like(e), e).clamp(min=-117)
    return torch.ldexp(x.to(_F32), -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    st, rnd = _State(), _Random(seed)
    st.case = case
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    if case["op"] == "requests":
        K, N, r, P = case["K"], case["N"], case["r"], case["pool"]
        lens = _rows(case)
        M = sum(lens)
        st.X, st.W = rnd.normal((M, K)), rnd.normal((N, K), K ** -0.5)
        st.A = ((rnd.uniform((P, r, K)) * 2 - 1) * K ** -0.5).to(_BF16)
        st.B = rnd.normal((P, N, r), 0.02)
        st.s = torch.tensor([0.5, 1.0, 2.0], device="cuda")[rnd.ints(0, 3, (P,))]
        st.ranks = torch.tensor([r, r // 2, r // 4], device="cuda", dtype=torch.int32)[rnd.ints(0, 3, (P,))] if case["mixed"] else None
        of = (P * rnd.uniform((len(lens),)) ** 2).to(torch.int32).clamp(max=P - 1)      # some tenants ask more often than others
        of = torch.where(rnd.uniform((len(lens),)) < 0.1, torch.full_like(of, -1), of)  # ... and some for the base model
        st.ids = torch.repeat_interleave(of, torch.tensor(lens, device="cuda"))
        st.Y, st.S = new((M, N), _BF16), new((M, r), _BF16)
    elif case["op"] == "norm_rope":
        M, H, G, D, rot = (case[k] for k in ("rows", "heads", "kv_heads", "dim", "rot"))
        st.qkv = rnd.normal((M, (H + 2 * G) * D))
        st.q = st.qkv[:, :H * D].view(M, H, D)
        st.k = st.qkv[:, H * D:(H + G) * D].view(M, G, D)
        st.gq, st.gk = rnd.normal((D,), 0.1, 1.0), rnd.normal((D,), 0.1, 1.0)
        per = -(-M // case["seqs"])
        if M <= 4 * case["seqs"]:                                    # decoding: anywhere in a context
            per, st.pos = 8192, rnd.ints(0, 8192, (M,)).to(torch.int32)
        else:                                                        # packed sequences
            st.pos = (torch.arange(M, device="cuda") % per).to(torch.int32)
        ang = torch.arange(per, device="cuda", dtype=_F64)[:, None] * 10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=_F64) / (rot // 2))
        st.cos, st.sin, st.eps = ang.cos().to(_F32), ang.sin().to(_F32), 1e-6
        st.dq_out = st.dk_out = None
        if case["do"] == "fwd":
            st.q_out, st.k_out = new((M, H, D), _BF16), new((M, G, D), _BF16)
        else:
            st.dq_out, st.dk_out = rnd.normal((M, H, D)), rnd.normal((M, G, D))
            st.dqkv = torch.zeros_like(st.qkv)                       # the values' part is attention's to write
            st.dq, st.dk = st.dqkv[:, :H * D].view(M, H, D), st.dqkv[:, H * D:(H + G) * D].view(M, G, D)
            st.dgq, st.dgk = new((D,), _F32), new((D,), _F32)
    elif case["op"] == "cache":
        M, G, D, page = (case[k] for k in ("rows", "kv_heads", "dim", "page"))
        pages = -(-M // page) + 8
        st.pages = _pages(rnd, pages, G, page, D, case["fp8"], filled=case["do"] == "read")
        at = rnd.permutation(pages)[:, None] * page + torch.arange(page, device="cuda")
        st.slots = at.reshape(-1)[:M].contiguous()
        if case["do"] == "write":
            spread = torch.exp(rnd.uniform((M, G, 1)) * 4 - 2)       # tokens and heads differ in magnitude
            st.kv = torch.stack((rnd.normal((M, G, D)) * spread, rnd.normal((M, G, D)) / spread), dim=1).to(_BF16)
        else:
            st.k_out, st.v_out = new((M, G, D), _BF16), new((M, G, D), _BF16)
    else:
        H, G, D, page = (case[k] for k in ("heads", "kv_heads", "dim", "page"))
        n, kv = _new_tokens(case), _kv_lens(case)
        used = [-(-v // page) for v in kv]
        pages = sum(used) + 4
        st.pages = _pages(rnd, pages, G, page, D, case["fp8"], filled=True)
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


def _pages(rnd, pages, G, page, D, fp8, filled):
    """(keys, values, key exponents, value exponents): [pages, heads, page, dim] and [pages, heads, page]."""
    shape = (pages, G, page, D)
    if not filled:
        k, v = (torch.zeros(shape, dtype=torch.float8_e4m3fn if fp8 else _BF16, device="cuda") for _ in range(2))
        return (k, v) + tuple(torch.zeros(shape[:3], dtype=torch.uint8, device="cuda") if fp8 else None for _ in range(2))
    k, v = rnd.normal(shape, 0.6), rnd.normal(shape)
    if not fp8:
        return k, v, None, None
    (k, ke), (v, ve) = _quantised(k), _quantised(v)
    return k, v, ke, ve


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    return {"requests": _run_requests, "norm_rope": _run_norm_rope, "cache": _run_cache, "attend": _run_attend}[st.case["op"]](st)


def _run_requests(st):
    if own:
        from paper_2510_00206_amd import binding
        return binding.lora_requests_fwd(st.X, st.W, st.A, st.B, st.ids, st.s, ranks=st.ranks, Y=st.Y, S=st.S)[0]
    X = st.X.to(_F32)
    g = st.ids.clamp(min=0)
    S = torch.bmm(st.A[g].to(_F32), X[:, :, None])[:, :, 0] * st.s[g][:, None]
    used = (st.ids >= 0)[:, None].expand_as(S)
    if st.ranks is not None:
        used = used & (torch.arange(S.shape[1], device=S.device)[None, :] < st.ranks[g][:, None])
    S = torch.where(used, S, torch.zeros_like(S))
    return (X @ st.W.to(_F32).t() + torch.bmm(st.B[g].to(_F32), S[:, :, None])[:, :, 0]).to(_BF16)


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


def _run_norm_rope(st):
    case = st.case
    if own:
        from paper_2510_00206_amd import binding
        kw = dict(eps=st.eps, interleaved=case["interleaved"])
        if case["do"] == "fwd":
            return binding.lora_qk_norm_rope_fwd(st.q, st.k, st.gq, st.gk, st.cos, st.sin, st.pos, q_out=st.q_out, k_out=st.k_out, **kw)
        return binding.lora_qk_norm_rope_bwd(st.q, st.k, st.gq, st.gk, st.cos, st.sin, st.pos, st.dq_out, st.dk_out, dq=st.dq, dk=st.dk,
                                             dgq=st.dgq, dgk=st.dgk, **kw)
    cos, sin = st.cos[st.pos.long()][:, None], st.sin[st.pos.long()][:, None]
    out = [], []
    for x, gamma, dy in ((st.q, st.gq, st.dq_out), (st.k, st.gk, st.dk_out)):
        x, gamma = x.to(_F32), gamma.to(_F32)
        inv = 1.0 / torch.sqrt(torch.mean(x * x, dim=-1, keepdim=True) + st.eps)
        n = x * inv
        if dy is None:
            out[0].append(_rotate(n * gamma, cos, sin, case["interleaved"]).to(_BF16))
            continue
        dn = _rotate(dy.to(_F32), cos, -sin, case["interleaved"])
        out[1].append(torch.sum(dn * n, dim=(0, 1)))
        dn = dn * gamma
        out[0].append((inv * (dn - n * torch.mean(dn * n, dim=-1, keepdim=True))).to(_BF16))
    return tuple(out[0] + out[1])


def _run_cache(st):
    k, v, ke, ve = st.pages
    if own:
        from paper_2510_00206_amd import binding
        cache = binding.KVCache(k, v, ke, ve)
        if st.case["do"] == "read":
            return binding.lora_kv_cache_read(cache, st.slots, k=st.k_out, v=st.v_out)
        binding.lora_kv_cache_write(cache, st.kv[:, 0], st.kv[:, 1], st.slots)
        return (k, v) if ke is None else (k, v, ke, ve)
    page, at = k.shape[2], (st.slots // k.shape[2], slice(None), st.slots % k.shape[2])
    if st.case["do"] == "read":
        return tuple((x[at].to(_F32) if e is None else torch.ldexp(x[at].to(_F32), e[at].to(torch.int32)[..., None] - 127)).to(_BF16)
                     for x, e in ((k, ke), (v, ve)))
    for x, e, new in ((k, ke, st.kv[:, 0]), (v, ve, st.kv[:, 1])):
        if e is None:
            x[at] = new
        else:
            codes, exps = _quantised(new)
            x.view(torch.uint8)[at] = codes.view(torch.uint8)
            e[at] = exps
    return (k, v) if ke is None else (k, v, ke, ve)


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
    K, V = ((x[st.table.long()].to(_F32) if e is None else torch.ldexp(x[st.table.long()].to(_F32), e[st.table.long()].to(torch.int32)[..., None] - 127))
            .transpose(1, 2).reshape(B, G, L, D) for x, e in ((k, ke), (v, ve)))
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
def work(case):
    if case["op"] == "requests":
        M, K, N, r, P = sum(_rows(case)), case["K"], case["N"], case["r"], case["pool"]
        # adapters in use: at most one to a request, and of a pool drawn with the square of a uniform number about so many
        n = len(_rows(case))
        used = sum(1.0 - (1.0 - (math.sqrt((g + 1) / P) - math.sqrt(g / P))) ** (0.9 * n) for g in range(P))
        mean_r = r * 7 / 12 if case["mixed"] else r
        return {"bytes": 2 * (M * K + N * K + M * N) + 2 * used * mean_r * (K + N), "flops": 2 * M * K * N + 2 * 0.9 * M * mean_r * (K + N)}
    if case["op"] == "norm_rope":
        M, H, D, rot = case["rows"], case["heads"] + case["kv_heads"], case["dim"], case["rot"]
        # in, out, (backward) the outputs' gradients; the rows of the tables that are in use
        return {"bytes": (2 if case["do"] == "fwd" else 3) * 2 * M * H * D + 4 * min(M, -(-M // case["seqs"])) * rot,
                "flops": (6 if case["do"] == "fwd" else 14) * M * H * D}
    if case["op"] == "cache":
        M, G, D = case["rows"], case["kv_heads"], case["dim"]
        return {"bytes": 2 * M * G * (2 * D + (D + 1 if case["fp8"] else 2 * D)) + 8 * M, "flops": 2 * 2 * M * G * D}
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    w = case["window"] or 1 << 40
    pairs = keys = 0
    for n, kv in zip(_new_tokens(case), _kv_lens(case)):
        pairs += sum(min(w, kv - n + i + 1) for i in range(n))
        keys += min(kv, w + n - 1)
    return {"bytes": 2 * 2 * sum(_new_tokens(case)) * H * D + 2 * keys * G * (D + 1 if case["fp8"] else 2 * D), "flops": 4 * pairs * H * D}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------
def _e4m3(x):
    """64-bit values rounded to the nearest with three fraction bits (ties to even), 2^-9 apart below 2^-6."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "requests":
        X = st.X.to(_F64)
        Y = X @ st.W.to(_F64).t()
        for g in torch.unique(st.ids).tolist():
            if g < 0:
                continue
            q = case["r"] if st.ranks is None else int(st.ranks[g])
            at = (st.ids == g).nonzero()[:, 0]
            Y[at] += float(st.s[g]) * ((X[at] @ st.A[g, :q].to(_F64).t()) @ st.B[g, :, :q].to(_F64).t())
        return Y
    if case["op"] == "norm_rope":
        half, inter = case["rot"] // 2, case["interleaved"]
        i = torch.arange(half, device="cuda")
        first, second = (2 * i, 2 * i + 1) if inter else (i, i + half)
        turn = torch.complex(st.cos.to(_F64), st.sin.to(_F64))[st.pos.long()][:, None, :]
        def turned(x, by):
            z = torch.complex(x[..., first], x[..., second]) * by
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y
        ys, dgs = [], []
        for x, gamma, dy in ((st.q, st.gq, st.dq_out), (st.k, st.gk, st.dk_out)):
            x, gamma = x.to(_F64), gamma.to(_F64)
            rms = (x.square().sum(-1, keepdim=True) / case["dim"] + st.eps).sqrt()
            if dy is None:
                ys.append(turned(x / rms * gamma, turn))
                continue
            up = turned(dy.to(_F64), turn.conj())
            dgs.append((up * x / rms).sum(0).sum(0))
            up = up * gamma
            ys.append(up / rms - x * (up * x).sum(-1, keepdim=True) / (case["dim"] * rms ** 3))
        return tuple(ys + dgs)
    k, v, ke, ve = st.pages
    page = k.shape[2]
    if case["op"] == "cache":
        p, o = st.slots // page, st.slots % page
        if case["do"] == "read":
            scale = lambda e: 1.0 if e is None else torch.exp2(e[p, :, o].to(_F64) - 127)[..., None]
            return k[p, :, o].to(_F32).to(_F64) * scale(ke), v[p, :, o].to(_F32).to(_F64) * scale(ve)
        out = [k.to(_F32).to(_F64), v.to(_F32).to(_F64)]
        for x, new in zip(out, (st.kv[:, 0].to(_F64), st.kv[:, 1].to(_F64))):
            if ke is not None:
                top = new.abs().amax(-1)
                e = torch.where(top > 0, torch.ceil(torch.log2(top / 448.0)), torch.zeros_like(top)).clamp(min=-117)
                new = _e4m3(new / torch.exp2(e)[..., None])
            x[p, :, o] = new
        return tuple(out) if ke is None else (out[0], out[1], None, None)
    if sum(_new_tokens(case)) * case["heads"] * case["kv_hi"] > 1 << 31:
        return None
    G, D = case["kv_heads"], case["dim"]
    out = torch.empty(st.q.shape, dtype=_F64, device="cuda")
    for b, (n, kv) in enumerate(zip(_new_tokens(case), _kv_lens(case))):
        pg = st.table[b, :-(-kv // page)].long()
        row = int(st.offsets[b])
        for g in range(G):
            Kg, Vg = (x[pg, g].to(_F32).to(_F64) * (1.0 if e is None else torch.exp2(e[pg, g].to(_F64) - 127)[..., None]) for x, e in ((k, ke), (v, ve)))
            Kg, Vg = Kg.reshape(-1, D)[:kv], Vg.reshape(-1, D)[:kv]
            i = torch.arange(kv - n, kv, device="cuda")[:, None] - torch.arange(kv, device="cuda")[None, :]
            seen = (i >= 0) & (i < (case["window"] or 1 << 40))
            for h in range(g * (case["heads"] // G), (g + 1) * (case["heads"] // G)):
                s = (st.q[row:row + n, h].to(_F64) @ Kg.t()) / math.sqrt(D)
                out[row:row + n, h] = torch.softmax(torch.where(seen, s, torch.full_like(s, -math.inf)), dim=-1) @ Vg
    return out
