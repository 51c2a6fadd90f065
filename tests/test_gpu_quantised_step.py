"""The operators of serving over 4 bits together, as examples/serving_step.py runs them after quantise(): chunks and decoding against the whole prompt in
64 bits, replays of captured steps, two of them over one workspace, a busy stream, several threads."""
import threading

import pytest
import torch

from examples.serving_step import AttentionBlock, Step
from paper_2510_00206_amd import binding
from quant_util import quantised4, widened4
from serve_util import BF16, F64, attention, gen, norm_rope, quantised, widened

pytestmark = pytest.mark.gpu
FORMS = ["bf16", "fp8", "fp4"]


def _block(**kw):
    return AttentionBlock(**{**dict(hidden=320, heads=4, kv_heads=2, dim=64, rank=16, adapters=5, positions=300, seed=3), **kw}).quantise()


def _cache(block, pages, form, page=16):
    return binding.KVCache.empty(pages, page, block.kv_heads, block.dim, fp8=form == "fp8", fp4=form == "fp4")


def _whole(block, x, adapter, form):
    """The block over a whole prompt in 64 bits, rounded to bf16 where the tensors between the calls are and, keys from 64 bits, to what the cache holds."""
    c = lambda t: t.cpu().to(F64)
    H, G, D = block.heads, block.kv_heads, block.dim

    def layer(x, w, held, a, b):
        codes, exps = quantised4(c(w))
        assert torch.equal(codes, held[0].cpu()) and torch.equal(exps, held[1].cpu())
        y = x @ widened4(codes, exps).t()
        if 0 <= adapter < a.shape[0]:
            r = int(block.ranks[adapter])
            y = y + ((float(block.scale[adapter]) * (x @ c(a[adapter, :r]).t())).to(BF16).to(F64)) @ c(b[adapter, :, :r]).t()
        return y.to(BF16).to(F64)
    qkv = layer(c(x), block.w_qkv, block.four_bits[0], block.a_qkv, block.b_qkv)
    n = x.shape[0]
    q, k, v = (qkv[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    q, k = (norm_rope(t, c(g), block.cos.cpu(), block.sin.cpu(), torch.arange(n), 1e-6, False)[0] for t, g in ((q, block.gamma_q), (k, block.gamma_k)))
    if form == "fp4":
        k, v = widened4(*quantised4(k)), widened4(*quantised4(v))
    elif form == "fp8":
        k, v = widened(*quantised(k)), widened(*quantised(v))
    else:
        k = k.to(BF16).to(F64)
    o, _ = attention(q.to(BF16).to(F64), k, v, n, n, D ** -0.5, 0)
    return layer(o.to(BF16).to(F64).flatten(1), block.w_out, block.four_bits[1], block.a_out, block.b_out)


@pytest.mark.parametrize("form", FORMS)
def test_chunks_and_decoding_equal_the_whole_prompt(form):
    """Two prompts with different adapters, a third without, in uneven chunks, then token by token, over pages in disorder.  Each side rounds the same values at
    the same places; a sum of 320 terms in fp32 is some 2^-20 off, so about one value in 2^11 falls on the other side of a step of bf16, and of the cache's
    entries (steps of 2^-2 of the value at 4 bits) those whose input moved by d, with a chance of d over the step: a mean square of d times the step, below
    (2^-10)^2.  The weights of attention are rounded to bf16 on one side only, and so the 2-norm of the difference stays within four roundings to bf16, eight
    where the cache is quantised."""
    block = _block()
    total = 45
    cache = _cache(block, 12, form)
    pages, adapters = [[7, 2, 9], [0, 11, 4], [5, 1, 10]], [3, 1, -1]
    g = gen(8)
    x = [torch.randn((total, 320), generator=g).to(BF16) for _ in pages]
    got = [[], [], []]
    for n, before in (((17, 30, 1), (0, 0, 0)), ((23, 5, 40), (17, 30, 1))) + tuple(((1, 1, 1), (40 + i, 35 + i, 41 + i)) for i in range(4)):
        step = Step(block, cache, n, total + 3, 3)
        step.plan(adapters, pages, before)
        out = block.serve(step, torch.cat([x[i][b:b + m] for i, (b, m) in enumerate(zip(before, n))]).cuda()).cpu()
        for i in range(3):
            got[i].append(out[int(step.offsets[i]):int(step.offsets[i + 1])])
    for i in range(3):
        rows = torch.cat(got[i]).to(F64)
        ref = _whole(block, x[i][:rows.shape[0]], adapters[i], form)
        off = float((rows - ref).norm() / ref.norm())
        print("serving over 4 bits", i, form, off, flush=True)
        assert off <= (4 if form == "bf16" else 8) * 2.0 ** -8


@pytest.mark.parametrize("form", FORMS)
def test_replays_of_captured_steps(form):
    """A decode step and a step of chunks in a HIP graph each, over the same cache and the same workspace, replayed in turn for longer and longer sequences, with eager
    steps of another cache between the replays: each replay as the eager step, bit for bit, and the caches the same at the end."""
    block = _block()
    pages = [[4 * i + j for j in range(4)] for i in range(6)]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    data = torch.randn((30, 12, 320), generator=g, device="cuda").to(BF16)
    eager, held = _cache(block, 24, form), _cache(block, 24, form)
    shapes = ([1] * 6, [7, 5])
    e, s = ([Step(block, cache, n, 64, 4) for n in shapes] for cache in (eager, held))
    small = min(s, key=lambda t: t.workspace.numel())
    small.workspace = max((t.workspace for t in s), key=lambda t: t.numel())
    other = Step(block, _cache(block, 24, form), [9, 33], 33, 4)
    other.plan([0, 2], pages[:2], [0, 0])
    x = [torch.zeros((sum(n), 320), dtype=BF16, device="cuda") for n in shapes]
    graphs = []
    for t, xi, n in zip(s, x, shapes):
        t.plan([0] * len(n), pages[:len(n)], [0] * len(n))
        block.serve(t, xi)                                  # first launches outside the capture
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            block.serve(t, xi)
    before = [0] * 6
    for n in range(14):
        for j, count in enumerate(shapes):
            rows = data[n, :sum(count)] if j == 0 else data[14 + n, :sum(count)]
            if j == 1 and n % 4:
                continue
            for t in (e[j], s[j]):
                t.plan([(n + i) % 6 - 1 for i in range(len(count))], pages[:len(count)], before[:len(count)])
            x[j].copy_(rows)
            s[j].out.fill_(7.0)
            want = block.serve(e[j], rows).clone()
            if n % 3 == 0:
                block.serve(other, torch.cat([data[n]] * 4)[:42])
            torch.cuda.synchronize()
            graphs[j].replay()
            torch.cuda.synchronize()
            assert torch.equal(s[j].out, want), (n, j)
            for i, m in enumerate(count):
                before[i] += m
    p = torch.tensor([a * 16 + b for i in range(6) for a in pages[i] for b in range(16) if 16 * (a % 4) + b < before[i]], device="cuda")
    for a, b in zip(eager.tensors, held.tensors):
        if a is not None:
            assert torch.equal(a[p // 16, :, p % 16].view(torch.uint8), b[p // 16, :, p % 16].view(torch.uint8))


def test_training_step():
    """Gradients of the projection over the widened weights, with norm and rotation, against autograd in 64 bits over what the codes hold (no dropout): within what the roundings
    to bf16 of qkv, its gradient and the saved S leave, four of them (2-norm); and a difference along dA and dB."""
    block = _block()
    H, G, D, M = 4, 2, 64, 50
    g = gen(4)
    draw = lambda *shape: torch.randn(shape, generator=g).to(BF16)
    x, dq, dk, dv = draw(M, 320), draw(M, H, D), draw(M, G, D), draw(M, G, D)
    pos = torch.randint(0, 300, (M,), generator=g, dtype=torch.int32)
    outs, grads = block.train(x.cuda(), pos.cuda(), dq.cuda(), dk.cuda(), dv.cuda(), adapter=2, dropout=0.0)
    c = lambda t: t.detach().cpu().to(F64).clone().requires_grad_()
    W = widened4(*(t.cpu() for t in block.four_bits[0]))
    leaves = X, A, B, gq, gk = c(x), c(block.a_qkv[2]), c(block.b_qkv[2]), c(block.gamma_q), c(block.gamma_k)

    def forward(X, A, B, gq, gk):
        qkv = X @ W.t() + 2.0 * ((X @ A.t()) @ B.t())
        q, k, v = (qkv[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        return *(norm_rope(t, gm, block.cos.cpu(), block.sin.cpu(), pos, 1e-6, False)[0] for t, gm in ((q, gq), (k, gk))), v
    ys = forward(*leaves)
    for got, ref in zip(outs, ys):
        assert float(((got.cpu().to(F64) - ref).norm() / ref.norm()).detach()) <= 4 * 2.0 ** -8
    weights = [t.to(F64) for t in (dq, dk, dv)]
    refs = torch.autograd.grad(ys, leaves, weights)
    for got, ref, name in zip(grads, refs, ("dx", "dA", "dB", "dgamma_q", "dgamma_k")):
        assert float((got.cpu().to(F64) - ref).norm() / ref.norm()) <= 4 * 2.0 ** -8, name
    loss = lambda A, B: sum((y * w).sum() for y, w in zip(forward(X, A, B, gq, gk), weights))
    with torch.no_grad():
        for i, got in ((1, grads[1].cpu().to(F64)), (2, grads[2].cpu().to(F64))):
            h = 1e-4 / float(got.norm())
            ends = [loss(*(t + (sign * h * got if j == i else 0) for j, t in ((1, A), (2, B)))) for sign in (1, -1)]
            slope = float(ends[0] - ends[1]) / (2 * h)
            assert abs(slope - float((refs[i] * got).sum())) <= 1e-4 * abs(slope) and abs(slope - float((got * got).sum())) <= 8 * 2.0 ** -8 * abs(slope)


def test_a_busy_stream():
    """All calls of a step wait for the work that its stream still has before them: launched anywhere else they would read zeros."""
    block = _block()
    x = torch.randn((40, 320), device="cuda").to(BF16)
    big = torch.randn((8192, 8192), device="cuda").to(BF16)
    out, spare, held = [], torch.empty_like(big), []
    stream = torch.cuda.Stream()
    for busy in (False, True):
        cache = _cache(block, 3, "fp4")
        step = Step(block, cache, [40], 40, 3)
        late, w, codes = torch.zeros_like(x), torch.zeros_like(block.w_out), tuple(torch.zeros_like(t) for t in block.four_bits[1])
        own = AttentionBlock.__new__(AttentionBlock)
        own.__dict__.update(block.__dict__)
        own.four_bits = block.four_bits[0], codes
        step.plan([2], [[0, 1, 2]], [0])
        positions = step.positions.clone()
        step.positions.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            ready = torch.cuda.Event()
            for _ in range(200 if busy else 0):             # some 170 ms, which the launches below take less than
                torch.mm(big, big, out=spare)
            late.copy_(x)
            w.copy_(block.w_out)
            step.positions.copy_(positions)
            ready.record()
            binding.lora_weights_write(w, *codes)
            out.append(own.serve(step, late).clone())
            held.append(binding.lora_kv_cache_read(cache, step.slots))
            back = binding.lora_weights_read(*codes)
            early = not ready.query()
        torch.cuda.synchronize()
        assert early or not busy, "the stream's work ended before the step was launched"
        assert torch.equal(back.cpu().to(F64), widened4(*(t.cpu() for t in block.four_bits[1])))
    assert torch.equal(out[0], out[1]) and all(torch.equal(a, b) for a, b in zip(*held)) and bool(held[0][0].abs().max() > 0)


def test_steps_from_several_threads():
    """Four threads, each with a stream, a cache and a step of its own size, at the same time: as one after the other."""
    block = _block()
    sizes = [[40], [1, 1, 1], [70, 2], [12]]
    x = [torch.randn((sum(n), 320), device="cuda").to(BF16) for n in sizes]

    def run(i, out, stream):
        with torch.cuda.stream(stream):
            for _ in range(20):
                step = Step(block, _cache(block, 20, FORMS[i % 3]), sizes[i], 80, 6)
                step.plan([2] * len(sizes[i]), [[6 * b + j for j in range(6)] for b in range(len(sizes[i]))], [0] * len(sizes[i]))
                out[i] = block.serve(step, x[i]).clone()
            stream.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    together, alone = [None] * 4, [None] * 4
    threads = [threading.Thread(target=run, args=(i, together, streams[i])) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(4):
        run(i, alone, streams[i])
    assert all(torch.equal(a, b) for a, b in zip(together, alone))
