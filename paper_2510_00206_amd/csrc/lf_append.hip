// What stands between the query/key/value projection and attention, in one pass: norms of queries and keys for each head (or none), their rotation by the
// row's position, queries out, keys and values into the slots of a paged cache (bf16, fp8 or 4 bits).
//   n = x / sqrt(mean(x^2) + eps);  y = R(gamma n)          (no norm: y = R(x))
// Queries, and keys of a bf16 cache: fp32, rounded once.  Keys that are quantised are formed in 64 bits and rounded once, from there (round_to_odd): next to a
// border of the quantiser's coarse steps a difference in the last bit of 32 gives another code, so that what is held would go by the order of a sum.
// Bound by HBM: 2 bytes an entry in, 2 a query entry out, what the cache's form takes of keys and values.  Against lora_qk_norm_rope_fwd and
// lora_kv_cache_write it spares a launch and the keys' way out and in again.  A wave for a row, or for a part of its heads, as in lf_rope.hip.
#include <algorithm>

#include "lf_rope_parts.h"

namespace lf {

constexpr int kAppendThreads = 256;

template <int GL>
__device__ __forceinline__ double sum_over_head(double v) {
#pragma unroll
    for (int o = GL / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

template <int GL, bool INTER>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs p) {
    const int64_t unit = (int64_t)blockIdx.x * (kAppendThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = unit / p.parts;
    if (row >= p.M) return;
    const int D = p.c.D, part = (int)(unit % p.parts);
    const RopeLane<GL, INTER> ln(D, p.rot);
    constexpr int HEADS = 64 / GL, U = 4;                      // heads of a pass; passes whose loads are in flight together
    const int of_q = (p.H + HEADS - 1) / HEADS, of_k = (p.c.heads + HEADS - 1) / HEADS;
    const int pos = p.pos[row];
    const int64_t slot = p.slots[row];
    const bool known = pos >= 0 && pos < p.positions, held = slot >= 0 && slot < p.c.pages << p.c.page_shift, norm = p.gamma_q != nullptr;
    float c[8], s[8];
    angles(p, ln, pos, known, c, s);
    auto gammas = [&](const lora_bf16* gamma, float (&g)[8], float (&o)[8]) {       // of this lane's entries and of the others of their pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = o[i] = 1.f;
        if (!norm) return;
        const u32x4 raw = gamma_of(gamma, ln);
        unpack8(raw, g);
        others(ln, raw, o);
    };
    // passes first, first + parts, .. of the heads at x_row
    auto heads = [&](const lora_bf16* x_row, int n, int passes, int first, auto&& take) {
        for (; first < passes; first += U * p.parts) {
            u32x4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = (first + u * p.parts) * HEADS + ln.slot;
                raw[u] = u32x4{0u, 0u, 0u, 0u};
                if (ln.active && head < n) raw[u] = *(const u32x4*)(x_row + (int64_t)head * D + 8 * ln.j);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int pass = first + u * p.parts, head = pass * HEADS + ln.slot;
                if (pass >= passes) break;
                take(raw[u], head, ln.active && head < n);
            }
        }
    };
    auto first_of = [&](int before) { const int r = (part - before) % p.parts; return r < 0 ? r + p.parts : r; };
    // norm and rotation in fp32
    auto turned = [&](u32x4 raw, const float (&cg)[8], const float (&sg)[8], float (&y)[8]) {
        float x[8], o[8], sum = 0.f;
        unpack8(raw, x);
        others(ln, raw, o);
        float inv = 1.f;
        if (norm) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
            inv = 1.f / sqrtf(sum_over_head<GL>(sum) / (float)D + p.eps);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = known ? inv * (x[i] * cg[i] + o[i] * sg[i]) : 0.f;
    };
    auto folded = [&](const lora_bf16* gamma, float (&cg)[8], float (&sg)[8]) {
        float g[8], o[8];
        gammas(gamma, g, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) { cg[i] = c[i] * g[i]; sg[i] = s[i] * o[i]; }
    };
    {
        float cg[8], sg[8];
        folded(p.gamma_q, cg, sg);
        heads(p.q + row * p.ldq, p.H, of_q, part, [&](u32x4 raw, int head, bool ok) {
            float y[8];
            turned(raw, cg, sg, y);
            if (ok) *(u32x4*)(p.q_out + row * p.ldqo + (int64_t)head * D + 8 * ln.j) = pack8(y);
        });
    }
    const int first_k = first_of(of_q);
    auto at_of = [&](int head, bool ok) { return ok ? head_of_slot(p.c, slot, head) : 0; };
    if (p.c.form == kCacheBf16) {
        float cg[8], sg[8];
        folded(p.gamma_k, cg, sg);
        heads(p.k + row * p.ldk, p.c.heads, of_k, first_k, [&](u32x4 raw, int head, bool ok) {
            float y[8];
            turned(raw, cg, sg, y);
            if (ok && held) *(u32x4*)((lora_bf16*)p.c.k + at_of(head, true) * D + 8 * ln.j) = pack8(y);
        });
    } else {
        double cg[8], sg[8];
        {
            float g[8], o[8];
            gammas(p.gamma_k, g, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) { cg[i] = (double)c[i] * (double)g[i]; sg[i] = (double)s[i] * (double)o[i]; }
        }
        heads(p.k + row * p.ldk, p.c.heads, of_k, first_k, [&](u32x4 raw, int head, bool ok) {
            float x[8], o[8], y[8];
            unpack8(raw, x);
            others(ln, raw, o);
            double inv = 1.0;
            if (norm) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += (double)x[i] * (double)x[i];
                inv = 1.0 / sqrt(sum_over_head<GL>(sum) / (double)D + (double)p.eps);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = known ? round_to_odd(inv * ((double)x[i] * cg[i] + (double)o[i] * sg[i])) : 0.f;
            hold_quantised<GL>(p.c, true, ok && held, at_of(head, ok && held), ln.j, y);
        });
    }
    heads(p.v + row * p.ldv, p.c.heads, of_k, first_of(of_q + of_k),
          [&](u32x4 raw, int head, bool ok) { hold_head<GL>(p.c, false, ok && held, at_of(head, ok && held), ln.j, raw); });
}

// Parts of a row: more than one while there are fewer rows than 16 waves to a compute unit.
hipError_t launch_append(AppendArgs a, bool interleaved, hipStream_t st) {
    return with_lanes(a.c.D, [&](auto gl) {
        constexpr int HEADS = 64 / gl();
        const int64_t all = (a.H + HEADS - 1) / HEADS + 2 * ((a.c.heads + HEADS - 1) / HEADS);
        a.parts = (int)std::min<int64_t>((16 * kComputeUnits + a.M - 1) / a.M, all);
        return with_pairs(interleaved, [&](auto inter) {
            // (a launch has fewer than 2^32 threads: 64 a row)
            constexpr int64_t ROWS = 1 << 25;
            hipError_t e = hipSuccess;
            for (int64_t left = a.M; left > 0 && e == hipSuccess; left -= ROWS) {
                a.M = std::min(left, ROWS);
                const int64_t blocks = (a.M * a.parts + kAppendThreads / 64 - 1) / (kAppendThreads / 64);
                hipLaunchKernelGGL((append_kernel<gl(), inter()>), dim3((unsigned)blocks), dim3(kAppendThreads), 0, st, a);
                e = hipGetLastError();
                a.q += a.M * a.ldq;
                a.k += a.M * a.ldk;
                a.v += a.M * a.ldv;
                a.q_out += a.M * a.ldqo;
                a.pos += a.M;
                a.slots += a.M;
            }
            return e;
        });
    });
}

}  // namespace lf
