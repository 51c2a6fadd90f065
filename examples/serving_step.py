"""The attention block of a decoder layer, with LoRA adapters on its projections: served to many tenants at once, and as a training step of one of
the adapters.

    python -m examples.serving_step            # 32 requests: prompts in chunks, then decoding; prints the time of a step

Serving: every row of a step is a token of some request, and names the request's adapter.  The fused query/key/value projection adds each row's
adapter (lora_requests_fwd), queries and keys are normalised and turned (lora_qk_norm_rope_fwd), keys and values go into the paged cache
(lora_kv_cache_write), the new tokens attend over it (lora_paged_attn_fwd), and the output projection takes the adapters again.  Prompts may come
in chunks, beside requests that decode: what a step needs to know of them are arrays on the GPU, so that a step of fixed size can be
captured in a HIP graph and replayed.
Serving over 4 bits (and training over the same weights, widened for the step): the same block after quantise(): both projections over 4-bit weights (lora_requests_quantised_fwd), queries, keys and values from the
projection to attention and the cache in one call (lora_kv_cache_append), which may be a 4-bit cache too.
Training: the same projection and norm with the backward passes of the library."""
import torch

from paper_2510_00206_amd import binding

BF16, I32 = torch.bfloat16, torch.int32


class AttentionBlock:
    """Weights of one layer and a pool of adapters: heads query heads and kv_heads key/value heads of `dim` entries."""

    def __init__(self, hidden, heads, kv_heads, dim, rank, adapters, positions=8192, seed=0, device="cuda"):
        self.heads, self.kv_heads, self.dim, self.rank = heads, kv_heads, dim, rank
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        normal = lambda shape, std, mean=0.0: (torch.randn(shape, generator=g, device=device) * std + mean).to(BF16)
        qkv, out = (heads + 2 * kv_heads) * dim, heads * dim
        self.w_qkv, self.w_out = normal((qkv, hidden), hidden ** -0.5), normal((hidden, out), out ** -0.5)
        # adapters of each projection: A [adapters, rank, in], B [adapters, out, rank], their scale and rank
        self.a_qkv, self.b_qkv = normal((adapters, rank, hidden), hidden ** -0.5), normal((adapters, qkv, rank), 0.02)
        self.a_out, self.b_out = normal((adapters, rank, out), out ** -0.5), normal((adapters, hidden, rank), 0.02)
        self.scale = torch.full((adapters,), 2.0, device=device)
        self.ranks = torch.tensor([rank if i % 2 == 0 else rank // 2 for i in range(adapters)], dtype=I32, device=device)
        self.gamma_q, self.gamma_k = normal((dim,), 0.1, 1.0), normal((dim,), 0.1, 1.0)
        angle = torch.arange(positions, device=device)[:, None] * 10000.0 ** (-torch.arange(dim // 2, device=device) / (dim // 2))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.four_bits = None

    def quantise(self):
        """4-bit weights from here on, in serving and (widened for the step) in training, so that adapters meet the weights that they are trained on.  -> the block"""
        self.four_bits = binding.lora_weights_write(self.w_qkv), binding.lora_weights_write(self.w_out)
        return self

    def serve(self, step, x):
        """x [tokens, hidden] of a Step -> the block's output [tokens, hidden]."""
        H, G, D = self.heads, self.kv_heads, self.dim
        if self.four_bits:
            return self._serve_four_bits(step, x)
        binding.lora_requests_fwd(x, self.w_qkv, self.a_qkv, self.b_qkv, step.adapters, self.scale, ranks=self.ranks, Y=step.qkv, S=step.s)
        q, k, v = (step.qkv[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        binding.lora_qk_norm_rope_fwd(q, k, self.gamma_q, self.gamma_k, self.cos, self.sin, step.positions, q_out=q, k_out=k)
        binding.lora_kv_cache_write(step.cache, k, v, step.slots)
        binding.lora_paged_attn_fwd(q, step.cache, step.table, step.offsets, step.lengths, step.max_new, step.max_length, out=step.mixed,
                                    workspace=step.workspace)
        return binding.lora_requests_fwd(step.mixed.flatten(1), self.w_out, self.a_out, self.b_out, step.adapters, self.scale, ranks=self.ranks,
                                         Y=step.out, S=step.s)[0]

    def _serve_four_bits(self, step, x):
        H, G, D = self.heads, self.kv_heads, self.dim
        qkv, out = self.four_bits
        binding.lora_requests_quantised_fwd(x, *qkv, self.a_qkv, self.b_qkv, step.adapters, self.scale, ranks=self.ranks, Y=step.qkv, S=step.s)
        q, k, v = (step.qkv[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        binding.lora_kv_cache_append(step.cache, q, k, v, self.cos, self.sin, step.positions, step.slots, self.gamma_q, self.gamma_k, q_out=q)
        binding.lora_paged_attn_fwd(q, step.cache, step.table, step.offsets, step.lengths, step.max_new, step.max_length, out=step.mixed,
                                    workspace=step.workspace)
        return binding.lora_requests_quantised_fwd(step.mixed.flatten(1), *out, self.a_out, self.b_out, step.adapters, self.scale, ranks=self.ranks,
                                                   Y=step.out, S=step.s)[0]

    def train(self, x, positions, dq, dk, dv, adapter=0, dropout=0.1, seed=1):
        """One adapter's forward and backward of the projection with norm and rotation, for the gradients dq, dk, dv that attention returns.
        -> (q, k, v), (dx, dA, dB, dgamma_q, dgamma_k)"""
        H, G, D = self.heads, self.kv_heads, self.dim
        a, b, s = self.a_qkv[adapter].contiguous(), self.b_qkv[adapter].contiguous(), float(self.scale[adapter])
        w = binding.lora_weights_read(*self.four_bits[0]) if self.four_bits else self.w_qkv
        qkv, saved = binding.lora_fwd(x, w, a, b, s, dropout, seed)
        part = lambda t: tuple(t[:, i * D:j * D].unflatten(1, (j - i, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        q, k, v = part(qkv)
        turned = binding.lora_qk_norm_rope_fwd(q, k, self.gamma_q, self.gamma_k, self.cos, self.sin, positions)
        d_qkv = torch.empty_like(qkv)
        pq, pk, pv = part(d_qkv)
        _, _, dgq, dgk = binding.lora_qk_norm_rope_bwd(q, k, self.gamma_q, self.gamma_k, self.cos, self.sin, positions, dq, dk, dq=pq, dk=pk)
        pv.copy_(dv)
        dx, da, db = binding.lora_bwd(x, w, a, b, saved, d_qkv, s, dropout, seed)
        return (*turned, v), (dx, da, db, dgq, dgk)


class Step:
    """What a step's calls take beside the weights: requests of `new` tokens each, whose tables and lengths are filled in by plan()."""

    def __init__(self, block, cache, new, max_length, pages_each, device="cuda"):
        tokens, seqs = sum(new), len(new)
        H, G, D = block.heads, block.kv_heads, block.dim
        empty = lambda shape, dtype=BF16: torch.empty(shape, dtype=dtype, device=device)
        self.cache, self.new, self.max_new, self.max_length = cache, list(new), max(new), max_length
        self.qkv, self.s = empty((tokens, (H + 2 * G) * D)), empty((tokens, block.rank))
        self.mixed, self.out = empty((tokens, H, D)), empty((tokens, block.w_out.shape[0]))
        self.adapters, self.positions, self.slots = empty((tokens,), I32), empty((tokens,), I32), empty((tokens,), torch.int64)
        self.table, self.lengths = torch.zeros((seqs, pages_each), dtype=I32, device=device), empty((seqs,), I32)
        self.offsets = torch.tensor([sum(new[:i]) for i in range(seqs + 1)], dtype=I32, device=device)
        self.workspace = binding.alloc_paged_attn_workspace(cache, tokens, H, seqs, self.max_new, max_length, device=device)

    def plan(self, adapters, pages, before):
        """adapters, before: of each request the adapter and the tokens that the cache holds already; pages: its page numbers."""
        page = self.cache.page
        rows = lambda values, dtype: torch.tensor(values, dtype=dtype)
        pos = [b + j for b, n in zip(before, self.new) for j in range(n)]
        of = [i for i, n in enumerate(self.new) for _ in range(n)]
        self.adapters.copy_(rows([adapters[i] for i in of], I32))
        self.positions.copy_(rows(pos, I32))
        self.slots.copy_(rows([pages[i][p // page] * page + p % page for i, p in zip(of, pos)], torch.int64))
        self.lengths.copy_(rows([b + n for b, n in zip(before, self.new)], I32))
        self.table.copy_(rows([list(p) + [0] * (self.table.shape[1] - len(p)) for p in pages], I32))


def serve(block, cache, label, requests=32, prompt=1000, decode=20):
    """Prompts four at a time in chunks of 250, then decoding, one token of every request a step; prints the time of such a step."""
    pages_each = cache.pages // requests
    pages = [list(range(i * pages_each, (i + 1) * pages_each)) for i in range(requests)]
    adapters = [i % 64 if i % 10 else -1 for i in range(requests)]
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    chunk = Step(block, cache, [250] * 4, prompt, pages_each)
    for first in range(0, requests, 4):
        for before in range(0, prompt, 250):
            ids = range(first, first + 4)
            chunk.plan([adapters[i] for i in ids], [pages[i] for i in ids], [before] * 4)
            block.serve(chunk, torch.randn((1000, 4096), generator=g, device="cuda").to(BF16))
    step = Step(block, cache, [1] * requests, prompt + decode, pages_each)
    x = torch.randn((requests, 4096), generator=g, device="cuda").to(BF16)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for n in range(decode):
        step.plan(adapters, pages, [prompt + n] * requests)
        begin.record()
        block.serve(step, x)
        end.record()
    torch.cuda.synchronize()
    print(f"attention block, {requests} requests, {prompt + decode} tokens each, {label}: {begin.elapsed_time(end) * 1e3:.0f} us a decode step; "
          f"output finite: {bool(torch.isfinite(step.out).all())}")


def main():
    block = AttentionBlock(hidden=4096, heads=32, kv_heads=8, dim=128, rank=16, adapters=64)
    pages = 32 * -(-1020 // 16)
    serve(block, binding.KVCache.empty(pages, 16, 8, 128, fp8=True), "fp8 cache")
    serve(block.quantise(), binding.KVCache.empty(pages, 16, 8, 128, fp4=True), "4-bit weights and cache")


if __name__ == "__main__":
    main()
