"""The operators around served adapters together, as examples/serving_step.py runs them: chunks and decoding against the whole prompt in 64 bits,
replays of a captured step against eager ones, a stream of its own, and the training step's gradients."""
import threading

import torch
import pytest

from examples.serving_step import AttentionBlock, Step
from paper_2510_00206_amd import binding
from serve_util import BF16, F64, attention, norm_rope, quantised, widened

pytestmark = pytest.mark.gpu


def _block(**kw):
    return AttentionBlock(**{**dict(hidden=320, heads=4, kv_heads=2, dim=64, rank=16, adapters=5, positions=300, seed=3), **kw})


def _whole(block, x, adapter, fp8):
    """The block over a whole prompt in 64 bits, rounded to bf16 (and e4m3) where the tensors between the calls are."""
    c = lambda t: t.cpu().to(F64)
    H, G, D = block.heads, block.kv_heads, block.dim

    def layer(x, w, a, b):
        y = x @ c(w).t()
        if 0 <= adapter < a.shape[0]:
            r = int(block.ranks[adapter])
            y = y + float(block.scale[adapter]) * ((x @ c(a[adapter, :r]).t()) @ c(b[adapter, :, :r]).t())
        return y.to(BF16).to(F64)
    qkv = layer(c(x), block.w_qkv, block.a_qkv, block.b_qkv)
    n = x.shape[0]
    q, k, v = (qkv[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    pos = torch.arange(n)
    q, k = (norm_rope(t, c(g), block.cos.cpu(), block.sin.cpu(), pos, 1e-6, False)[0].to(BF16) for t, g in ((q, block.gamma_q), (k, block.gamma_k)))
    if fp8:
        k, v = widened(*quantised(k)), widened(*quantised(v.to(BF16)))
    o, _ = attention(q.to(F64), k.to(F64), v.to(F64), n, n, D ** -0.5, 0)
    return layer(o.to(BF16).to(F64).flatten(1), block.w_out, block.a_out, block.b_out)


@pytest.mark.parametrize("fp8", [False, True])
def test_chunks_and_decoding_equal_the_whole_prompt(fp8):
    """Two prompts with different adapters (and a third without) in uneven chunks, then token by token, over pages in disorder.  Rounding of the
    tensors between the calls differs by what a unit of bf16 (e4m3) does where a value falls on the other side of a step: the 2-norm of the difference
    stays within four roundings to bf16 (and, a few values in a thousand on the other side of an e4m3 step, 2^-4 of them, as much again)."""
    block = _block()
    page, total = 16, 45
    cache = binding.KVCache.empty(12, page, block.kv_heads, block.dim, fp8)
    pages, adapters = [[7, 2, 9], [0, 11, 4], [5, 1, 10]], [3, 1, -1]
    g = torch.Generator()
    g.manual_seed(8)
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
        ref = _whole(block, x[i][:rows.shape[0]], adapters[i], fp8)
        off = float((rows - ref).norm() / ref.norm())
        print("serving step", i, fp8, off, flush=True)
        assert off <= (8 if fp8 else 4) * 2.0 ** -8


def test_replays_of_a_captured_step():
    """A decode step of fixed size in a HIP graph: replayed for longer and longer sequences, with eager steps of other sizes between the replays."""
    block = _block()
    total, page = 64, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    data = torch.randn((40, 6, 320), generator=g, device="cuda").to(BF16)
    pages = [[4 * i + j for j in range(4)] for i in range(6)]

    def caches():
        return binding.KVCache.empty(24, page, block.kv_heads, block.dim, True)
    eager, graph_cache = caches(), caches()
    e, s = Step(block, eager, [1] * 6, total, 4), Step(block, graph_cache, [1] * 6, total, 4)
    other = Step(block, caches(), [9, 33], 33, 4)
    other.plan([0, 2], pages[:2], [0, 0])
    x = torch.zeros((6, 320), dtype=BF16, device="cuda")
    s.plan([0, 1, 2, 3, 4, -1], pages, [0] * 6)
    block.serve(s, x)                                      # first launches outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.serve(s, x)
    for n in range(40):
        for t in (e, s):
            t.plan([n % 5, 1, 2, 3, (n + 1) % 5, -1], pages, [n] * 6)
        x.copy_(data[n])
        s.out.fill_(7.0)
        want = block.serve(e, data[n]).clone()
        if n % 3 == 0:
            block.serve(other, torch.cat([data[n]] * 7))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.out, want), n
    for a, b in zip(eager.tensors, graph_cache.tensors):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_a_stream_of_its_own():
    """The calls go to the stream that is current: a step on another one waits for what that stream was told to wait for, and only for it."""
    block = _block()
    pages = [[0, 1, 2]]
    x = torch.randn((40, 320), device="cuda").to(BF16)
    out = []
    for side in (False, True):
        cache = binding.KVCache.empty(3, 16, block.kv_heads, block.dim)
        step = Step(block, cache, [40], 40, 3)
        step.plan([2], pages, [0])
        if side:
            stream = torch.cuda.Stream()
            late = torch.zeros_like(x)
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                late.copy_(x)
                out.append(block.serve(step, late).clone())
            torch.cuda.current_stream().wait_stream(stream)
        else:
            out.append(block.serve(step, x).clone())
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1])


def test_a_busy_stream():
    """All calls of a step wait for the work that its stream still has before them: launched anywhere else they would read zeros."""
    block = _block()
    x = torch.randn((40, 320), device="cuda").to(BF16)
    big = torch.randn((8192, 8192), device="cuda").to(BF16)
    out, spare = [], torch.empty_like(big)
    stream = torch.cuda.Stream()
    for busy in (False, True):
        cache = binding.KVCache.empty(3, 16, block.kv_heads, block.dim, True)
        step = Step(block, cache, [40], 40, 3)
        late, positions, adapters = torch.zeros_like(x), torch.zeros_like(step.positions), torch.zeros_like(step.adapters)
        step.plan([2], [[0, 1, 2]], [0])
        for mine, right in ((positions, "positions"), (adapters, "adapters")):
            mine.copy_(getattr(step, right))
            getattr(step, right).zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            ready = torch.cuda.Event()
            for _ in range(200 if busy else 0):             # some 170 ms, which the launches below take less than
                torch.mm(big, big, out=spare)
            late.copy_(x)
            step.positions.copy_(positions)
            step.adapters.copy_(adapters)
            ready.record()
            out.append(block.serve(step, late).clone())
            early = not ready.query()
        torch.cuda.synchronize()
        assert early or not busy, "the stream's work ended before the step was launched"
    assert torch.equal(out[0], out[1])


def test_steps_from_several_threads():
    """Four threads, each with a stream, a cache and a step of its own size, at the same time: as one after the other."""
    block = _block()
    sizes = [[40], [1, 1, 1], [70, 2], [12]]
    x = [torch.randn((sum(n), 320), device="cuda").to(BF16) for n in sizes]

    def run(i, out, stream):
        with torch.cuda.stream(stream):
            for k in range(20):
                cache = binding.KVCache.empty(20, 16, block.kv_heads, block.dim, bool(i % 2))
                step = Step(block, cache, sizes[i], 80, 6)
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


def test_training_step():
    """Gradients of the projection with norm and rotation against autograd in 64 bits (no dropout): within what the roundings to bf16 of qkv, its
    gradient and the saved S leave, four of them (2-norm)."""
    block = _block()
    H, G, D, M = 4, 2, 64, 50
    g = torch.Generator()
    g.manual_seed(4)
    draw = lambda *shape: torch.randn(shape, generator=g).to(BF16)
    x, dq, dk, dv = draw(M, 320), draw(M, H, D), draw(M, G, D), draw(M, G, D)
    pos = torch.randint(0, 300, (M,), generator=g, dtype=torch.int32)
    outs, grads = block.train(x.cuda(), pos.cuda(), dq.cuda(), dk.cuda(), dv.cuda(), adapter=2, dropout=0.0)
    c = lambda t: t.detach().cpu().to(F64).clone().requires_grad_()
    X, A, B, gq, gk = c(x), c(block.a_qkv[2]), c(block.b_qkv[2]), c(block.gamma_q), c(block.gamma_k)
    qkv = X @ block.w_qkv.cpu().to(F64).t() + 2.0 * ((X @ A.t()) @ B.t())
    q, k, v = (qkv[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    yq, yk = (norm_rope(t, gm, block.cos.cpu(), block.sin.cpu(), pos, 1e-6, False)[0] for t, gm in ((q, gq), (k, gk)))
    for got, ref in zip(outs, (yq, yk, v)):
        assert float(((got.cpu().to(F64) - ref).norm() / ref.norm()).detach()) <= 4 * 2.0 ** -8
    refs = torch.autograd.grad([yq, yk, v], [X, A, B, gq, gk], [t.to(F64) for t in (dq, dk, dv)])
    for got, ref, name in zip(grads, refs, ("dx", "dA", "dB", "dgamma_q", "dgamma_k")):
        off = float((got.cpu().to(F64) - ref.detach()).norm() / ref.detach().norm())
        print("training step", name, off, flush=True)
        assert off <= 4 * 2.0 ** -8, name


def test_example_runs(capsys):
    from examples import serving_step
    serving_step.main()
    assert "output finite: True" in capsys.readouterr().out
