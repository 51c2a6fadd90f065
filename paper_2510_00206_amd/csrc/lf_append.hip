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

// Loads of U passes (every `parts`-th from `first` on, HEADS heads each) of the n heads at x_row, then take(raw, head, whether the lane has one) for each.
template <int GL, bool INTER, int U, class F>
__device__ __forceinline__ void by_passes(const RopeLane<GL, INTER>& ln, const lora_bf16* x_row, int n, int D, int passes, int first, int parts, F&& take) {
    constexpr int HEADS = 64 / GL;
    for (; first < passes; first += U * parts) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int head = (first + u * parts) * HEADS + ln.slot;
            raw[u] = u32x4{0u, 0u, 0u, 0u};
            if (ln.active && head < n) raw[u] = *(const u32x4*)(x_row + (int64_t)head * D + 8 * ln.j);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pass = first + u * parts, head = pass * HEADS + ln.slot;
            if (pass >= passes) break;
            take(raw[u], head, ln.active && head < n);
        }
    }
}

// The first workgroups have the keys' and values' waves, the others the queries': a wave for a row, or for a part of its heads.
template <int GL, bool INTER, bool WIDE>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs p) {
    constexpr int WAVES = kAppendThreads / 64, HEADS = 64 / GL, U = 4;
    const bool queries = (int)blockIdx.x >= p.kv_blocks;
    const int parts = queries ? p.parts : p.kv_parts, D = p.c.D;
    const int64_t unit = (int64_t)((int)blockIdx.x - (queries ? p.kv_blocks : 0)) * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = unit / parts;
    if (row >= p.M) return;
    const int part = (int)(unit % parts);
    const RopeLane<GL, INTER> ln(D, p.rot);
    const int pos = p.pos[row];
    const bool known = pos >= 0 && pos < p.positions, norm = p.gamma_q != nullptr;
    float c[8], s[8];
    auto folded = [&](const lora_bf16* gamma) {                // cosine and sine times gamma, of this lane's entries and of the others of their pairs
        angles(p, ln, pos, known, c, s);
        if (!norm) return;
        float g[8], o[8];
        const u32x4 raw = gamma_of(gamma, ln);
        unpack8(raw, g);
        others(ln, raw, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] *= g[i]; s[i] *= o[i]; }
    };
    auto turned = [&](u32x4 raw) {                             // norm and rotation in fp32
        float x[8], o[8], y[8], sum = 0.f;
        unpack8(raw, x);
        others(ln, raw, o);
        float inv = 1.f;
        if (norm) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
            inv = 1.f / sqrtf(sum_over_head<GL>(sum) / (float)D + p.eps);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = known ? inv * (x[i] * c[i] + o[i] * s[i]) : 0.f;
        return pack8(y);
    };
    if (queries) {
        folded(p.gamma_q);
        by_passes<GL, INTER, U>(ln, p.q + row * p.ldq, p.H, D, (p.H + HEADS - 1) / HEADS, part, parts, [&](u32x4 raw, int head, bool ok) {
            const u32x4 y = turned(raw);
            if (ok) *(u32x4*)(p.q_out + row * p.ldqo + (int64_t)head * D + 8 * ln.j) = y;
        });
        return;
    }
    const int passes = (p.c.heads + HEADS - 1) / HEADS;
    const int64_t slot = p.slots[row];
    const bool held = slot >= 0 && slot < p.c.pages << p.c.page_shift;
    auto at_of = [&](int head, bool to) { return to ? head_of_slot(p.c, slot, head) : 0; };
    by_passes<GL, INTER, WIDE ? 1 : 2>(ln, p.v + row * p.ldv, p.c.heads, D, passes, part, parts,
                            [&](u32x4 raw, int head, bool ok) { hold_head<GL>(p.c, false, ok && held, at_of(head, ok && held), ln.j, raw); });
    if constexpr (!WIDE) {
        folded(p.gamma_k);
        by_passes<GL, INTER, WIDE ? 1 : 2>(ln, p.k + row * p.ldk, p.c.heads, D, passes, part, parts, [&](u32x4 raw, int head, bool ok) {
            const u32x4 y = turned(raw);
            if (ok && held) *(u32x4*)((lora_bf16*)p.c.k + at_of(head, true) * D + 8 * ln.j) = y;
        });
    } else {
        angles(p, ln, pos, known, c, s);
        const u32x4 gamma = norm ? gamma_of(p.gamma_k, ln) : u32x4{0u, 0u, 0u, 0u};
        by_passes<GL, INTER, WIDE ? 1 : 2>(ln, p.k + row * p.ldk, p.c.heads, D, passes, part, parts, [&](u32x4 raw, int head, bool ok) {
            // (entry by entry: eight of them side by side take 139 registers, which every wave of the launch would have to hold)
            float x[8], o[8], y[8];
            unpack8(raw, x);
            double inv = 1.0;
            if (norm) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += (double)x[i] * (double)x[i];
                inv = 1.0 / sqrt(sum_over_head<GL>(sum) / (double)D + (double)p.eps);
            }
            others(ln, raw, o);
            float g[8], go[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = go[i] = 1.f;
            if (norm) {
                unpack8(gamma, g);
                others(ln, gamma, go);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                float ci = c[i], si = s[i], gi = g[i], goi = go[i];
                asm volatile("" : "+v"(ci), "+v"(si), "+v"(gi), "+v"(goi));       // (widened here, not once for all passes)
                y[i] = known ? round_to_odd(inv * ((double)x[i] * (double)gi * (double)ci + (double)o[i] * (double)goi * (double)si)) : 0.f;
            }
            __builtin_amdgcn_sched_barrier(0);
            hold_quantised<GL>(p.c, true, ok && held, at_of(head, ok && held), ln.j, y);
        });
    }
}

// Parts of a row.  Queries: of two passes, beside a quantised cache (whose keys take longer) four, and of one in small batches; keys and values: one part, in small batches
// one to a pass.  us in a captured graph, 32 + 2 x 8 heads of 128 (eight passes of queries, two of keys), parts of queries / of keys and values 1/1, 2/1, 4/1, 4/2, 8/2:
//   to 4 bits  16 rows 6.9, 6.9, 6.9, 4.8, 4.8;  800 9.4, 9.6, 9.7, 7.9, 8.8;  2085 14.8, 14.5, 14.6, 15.0, 17.2;  8192 46.4, 46.0, 51.2, 53.5, 66.4
//   to fp8     16 rows 7.3, 7.2, 7.2, 5.0, 5.0;  800 9.9, 10.1, 10.2, 8.1, 8.9;  2085 15.0, 14.5, 14.5, 15.4, 17.4;  8192 47.4, 47.3, 52.1, 54.9, 67.5
//   bf16       16 rows 6.2, 4.4, 4.2, 3.6, 3.6;  800 8.9, 7.6, 6.8, 7.1, 8.1;  2085 12.8, 12.5, 11.9, 12.5, 14.0;  8192 46.5, 44.1, 44.7, 47.7, 55.4
// This rule: 4.8, 7.8, 14.3, 46.4; 5.0, 8.1, 14.4, 47.1; 3.6, 7.1, 11.9, 45.1.  (The bf16 kernel with the cache's form a constant in it too: 2085 rows 12.6 instead of 12.0.)
hipError_t launch_append(AppendArgs a, bool interleaved, hipStream_t st) {
    return with_lanes(a.c.D, [&](auto gl) {
        constexpr int HEADS = 64 / gl(), WAVES = kAppendThreads / 64;
        const int64_t of_q = (a.H + HEADS - 1) / HEADS, of_k = (a.c.heads + HEADS - 1) / HEADS, each = a.c.form == kCacheBf16 ? 2 : 4;
        const auto few = [&](int waves) { return (waves * kComputeUnits + a.M - 1) / a.M; };       // parts that make so many waves to a compute unit
        a.parts = (int)std::min(std::max((of_q + each - 1) / each, few(12)), of_q);
        a.kv_parts = (int)std::min(few(4), of_k);
        return with_pairs(interleaved, [&](auto inter) {
            // (a launch has fewer than 2^32 threads, and these are up to 64 a pass)
            const int64_t ROWS = std::max<int64_t>((1ll << 25) / (a.parts + a.kv_parts), 1);
            hipError_t e = hipSuccess;
            for (int64_t left = a.M; left > 0 && e == hipSuccess; left -= ROWS) {
                a.M = std::min(left, ROWS);
                a.kv_blocks = (int)((a.M * a.kv_parts + WAVES - 1) / WAVES);
                const unsigned blocks = (unsigned)(a.kv_blocks + (a.M * a.parts + WAVES - 1) / WAVES);
                if (a.c.form == kCacheBf16) hipLaunchKernelGGL((append_kernel<gl(), inter(), false>), dim3(blocks), dim3(kAppendThreads), 0, st, a);
                else hipLaunchKernelGGL((append_kernel<gl(), inter(), true>), dim3(blocks), dim3(kAppendThreads), 0, st, a);
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
