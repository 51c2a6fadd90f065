// Norms of queries and keys for each head with the rotation by the row's position in the same pass, and its backward.
//   forward    n = x / rms,  rms = sqrt(mean(x^2) + eps);  y = R(gamma n)
//   backward   e = R^T dy;  dgamma = sum e n;  u = gamma e;  dx = (u - n mean(u n)) / rms
// R turns pairs of the head's first `rot` entries by the angles of its position.  x is read once (backward: x and dy), statistics are
// fp32, the result is rounded once.  Bound by HBM: 4 (6) bytes an element.  Eight entries to a lane (16-byte loads), 8, 16 or
// 32 lanes to a head by its size; a head's sums are butterflies over its lanes.  With R's cosines and sines multiplied by gamma once per
// row, y is one product and one multiply-add an entry; a pair's other entry comes from the lane that holds it, as the bf16 it was.
// Outputs are ordinary stores.  Past the caches the kernels themselves are faster, their reader is slower by more: us, stored / past the caches, alone and with
// the reading of the outputs behind, three sets in turn, 32 + 8 heads of 128: forward, 2048 rows (21 MB) 12.7 / 11.1, 21.4 / 21.5; 8192 (84 MB) 39.3 / 34.3, 69.5 / 71.6;
// 32768 (336 MB) 130.6 / 122.9, 241.7 / 252.4; backward, 4096 rows 34.8 / 30.8, 53.8 / 55.4; 8192 58.2 / 55.3, 95.5 / 94.7; 16384 105.4 / 99.5, 173.0 / 180.8.
// Measured (a copy of 2 GiB runs at 4.9 TB/s): forward, 8192 rows of 32 + 8 heads of 128, 168 MB, 38.7 us, 4.3 TB/s; backward, 5003 rows of 64 + 8, 277 MB, 61 us,
// 4.7 of them the sum of its planes; forward of 16 rows 4 us: the launch, and position, table and row read one after the other.
#include <algorithm>

#include "lf_serve.h"

namespace lf {

constexpr int kRopeThreads = 256;
// The backward: each workgroup leaves a plane of partial sums, so no more than the registers let run at once, four on every compute unit, of four waves, or
// (32 lanes to a head) three.  us, of 4 / 8 / 16 waves: 5003 rows of 64 + 8 heads 60.9 / 63.6 / 65.5, 16000 rows of 32 + 8 100 / 105 / 105.
constexpr int kRopeBlocks = 4 * kComputeUnits;
constexpr int rope_bwd_waves(int lanes) { return lanes == 32 ? 3 : 4; }

// GL lanes to a head, a wave for a row, or for a part of its heads.
template <int GL, bool INTER>
struct RopeLane {
    int j, slot;                       // lane of the head, head of the wave
    bool active, turned;               // ... has entries; they are in the rotated part
    int at, other;                     // first index into a row of the tables; wave lane with the other entries of this one's pairs
    float sign;                        // of the sine in y: - for the first entry of a pair
    __device__ __forceinline__ RopeLane(int D, int rot) {
        const int l = threadIdx.x & 63;
        j = l % GL;
        slot = l / GL;
        active = 8 * j < D;
        turned = 8 * j < rot;
        const bool first = INTER || 8 * j < rot / 2;
        at = INTER ? 4 * j : first ? 8 * j : 8 * j - rot / 2;
        other = INTER || !turned ? l : first ? l + rot / 16 : l - rot / 16;
        sign = first ? -1.f : 1.f;
    }
};

template <int GL>
__device__ __forceinline__ float sum_over_head(float v) {
#pragma unroll
    for (int o = GL / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Cosine and (signed) sine of each of a lane's entries.
template <int GL, bool INTER>
__device__ __forceinline__ void angles(const RopeArgs& p, const RopeLane<GL, INTER>& ln, int pos, bool known, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
    if (!ln.turned || !known) return;
    const float* cr = p.cos_ + (int64_t)pos * (p.rot / 2) + ln.at;
    const float* sr = p.sin_ + (int64_t)pos * (p.rot / 2) + ln.at;
    if constexpr (INTER) {
        const f32x4 cv = *(const f32x4*)cr, sv = *(const f32x4*)sr;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = cv[i / 2]; s[i] = i & 1 ? sv[i / 2] : -sv[i / 2]; }
    } else {
        const f32x4 c0 = *(const f32x4*)cr, c1 = *(const f32x4*)(cr + 4), s0 = *(const f32x4*)sr, s1 = *(const f32x4*)(sr + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = i < 4 ? c0[i & 3] : c1[i & 3]; s[i] = ln.sign * (i < 4 ? s0[i & 3] : s1[i & 3]); }
    }
}

// The other entries of this lane's pairs.
template <int GL, bool INTER>
__device__ __forceinline__ void others(const RopeLane<GL, INTER>& ln, u32x4 raw, float (&o)[8]) {
    if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = raw[i] >> 16 | raw[i] << 16;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = __shfl(raw[i], ln.other);
    }
    unpack8(raw, o);
}

template <int GL, bool INTER>
__device__ __forceinline__ u32x4 gamma_of(const lora_bf16* g, const RopeLane<GL, INTER>& ln) {
    u32x4 v = u32x4{0u, 0u, 0u, 0u};
    if (ln.active) v = *(const u32x4*)(g + 8 * ln.j);
    return v;
}

// A wave's row is done in passes of 64 / GL heads, first the queries' passes, then the keys'; part i of the row takes passes i, i + parts, ..
template <int GL>
struct RopePasses {
    static constexpr int HEADS = 64 / GL;
    int of_q, all;
    // first of the keys' passes that part `part` takes
    __device__ __forceinline__ int first_k(int part, int parts) const { const int r = (part - of_q) % parts; return r < 0 ? r + parts : r; }
    __host__ __device__ RopePasses(int H, int G) : of_q((H + HEADS - 1) / HEADS), all((H + HEADS - 1) / HEADS + (G + HEADS - 1) / HEADS) {}
};

template <int GL, bool INTER>
__global__ void __launch_bounds__(kRopeThreads) rope_fwd_kernel(RopeArgs p) {
    const int64_t unit = (int64_t)blockIdx.x * (kRopeThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = unit / p.parts;
    if (row >= p.M) return;
    const RopeLane<GL, INTER> ln(p.D, p.rot);
    const RopePasses<GL> ps(p.H, p.G);
    const int pos = p.pos[row];
    const bool known = pos >= 0 && pos < p.positions;
    float cq[8], sq[8], ck[8], sk[8];
    {
        float c[8], s[8], g[8], o[8];
        angles(p, ln, pos, known, c, s);
        auto fold = [&](const lora_bf16* gamma, float (&cg)[8], float (&sg)[8]) {
            const u32x4 raw = gamma_of(gamma, ln);
            unpack8(raw, g);
            others(ln, raw, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) { cg[i] = c[i] * g[i]; sg[i] = s[i] * o[i]; }
        };
        fold(p.gamma_q, cq, sq);
        fold(p.gamma_k, ck, sk);
    }
    auto heads = [&](const lora_bf16* x_row, lora_bf16* out_row, int n, int passes, int first, const float (&cg)[8], const float (&sg)[8]) {
        constexpr int U = 4;                               // passes whose loads are in flight together
        for (; first < passes; first += U * p.parts) {
            u32x4 raw[U];
            bool ok[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int head = (first + u * p.parts) * ps.HEADS + ln.slot;
                ok[u] = ln.active && head < n;
                raw[u] = u32x4{0u, 0u, 0u, 0u};
                if (ok[u]) raw[u] = *(const u32x4*)(x_row + (int64_t)head * p.D + 8 * ln.j);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int pass = first + u * p.parts;
                if (pass >= passes) break;
                float x[8], o[8], y[8], sum = 0.f;
                unpack8(raw[u], x);
                others(ln, raw[u], o);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
                const float inv = 1.f / sqrtf(sum_over_head<GL>(sum) / (float)p.D + p.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = inv * (x[i] * cg[i] + o[i] * sg[i]);
                u32x4 out = pack8(y);
                if (!known) out = u32x4{0u, 0u, 0u, 0u};
                if (ok[u]) *(u32x4*)(out_row + (int64_t)(pass * ps.HEADS + ln.slot) * p.D + 8 * ln.j) = out;
            }
        }
    };
    const int part = (int)(unit % p.parts);
    heads(p.q + row * p.ldq, p.q_out + row * p.ldqo, p.H, ps.of_q, part, cq, sq);
    heads(p.k + row * p.ldk, p.k_out + row * p.ldko, p.G, ps.all - ps.of_q, ps.first_k(part, p.parts), ck, sk);
}

template <int GL, bool INTER>
__global__ void __launch_bounds__(64 * rope_bwd_waves(GL), rope_bwd_waves(GL)) rope_bwd_kernel(RopeArgs p) {
    constexpr int WAVES = rope_bwd_waves(GL);
    __shared__ float red[WAVES][2][GL * 8];
    const RopeLane<GL, INTER> ln(p.D, p.rot);
    const RopePasses<GL> ps(p.H, p.G);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float dgq[8], dgk[8];
    const u32x4 gq = gamma_of(p.gamma_q, ln), gk = gamma_of(p.gamma_k, ln);
#pragma unroll
    for (int i = 0; i < 8; ++i) dgq[i] = dgk[i] = 0.f;
    const int64_t units = p.M * p.parts;
    for (int64_t unit = (int64_t)blockIdx.x * WAVES + w; unit < units; unit += (int64_t)gridDim.x * WAVES) {
        const int64_t row = unit / p.parts;
        const int pos = p.pos[row];
        const bool known = pos >= 0 && pos < p.positions;
        float c[8], s[8];
        angles(p, ln, pos, known, c, s);
        auto heads = [&](const lora_bf16* x_row, const lora_bf16* dy_row, lora_bf16* out_row, int n, int passes, int first, u32x4 gamma,
                         float (&dg)[8]) {
            float g[8];
            unpack8(gamma, g);
            constexpr int U = 2;
            for (; first < passes; first += U * p.parts) {
                u32x4 xr[U], dr[U];
                bool ok[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int head = (first + u * p.parts) * ps.HEADS + ln.slot;
                    ok[u] = ln.active && head < n;
                    xr[u] = dr[u] = u32x4{0u, 0u, 0u, 0u};
                    if (ok[u] && known) {                  // (a row outside the tables may hold infinities and NaN, and 0 times those is NaN)
                        xr[u] = *(const u32x4*)(x_row + (int64_t)head * p.D + 8 * ln.j);
                        dr[u] = *(const u32x4*)(dy_row + (int64_t)head * p.D + 8 * ln.j);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int pass = first + u * p.parts;
                    if (pass >= passes) break;
                    float x[8], e[8], o[8], sxx = 0.f, sux = 0.f;
                    unpack8(xr[u], x);
                    unpack8(dr[u], e);
                    others(ln, dr[u], o);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        e[i] = e[i] * c[i] - o[i] * s[i];
                        sxx += x[i] * x[i];
                        sux += e[i] * g[i] * x[i];
                    }
                    sxx = sum_over_head<GL>(sxx);
                    sux = sum_over_head<GL>(sux);
                    const float inv = 1.f / sqrtf(sxx / (float)p.D + p.eps), back = inv * inv * sux / (float)p.D;
                    float dx[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        dg[i] += e[i] * x[i] * inv;
                        dx[i] = inv * (e[i] * g[i] - x[i] * back);
                    }
                    u32x4 out = pack8(dx);
                    if (!known) out = u32x4{0u, 0u, 0u, 0u};
                    if (ok[u]) *(u32x4*)(out_row + (int64_t)(pass * ps.HEADS + ln.slot) * p.D + 8 * ln.j) = out;
                }
            }
        };
        const int part = (int)(unit % p.parts);
        heads(p.q + row * p.ldq, p.dq_out + row * p.lddq, p.q_out + row * p.ldqo, p.H, ps.of_q, part, gq, dgq);
        heads(p.k + row * p.ldk, p.dk_out + row * p.lddk, p.k_out + row * p.ldko, p.G, ps.all - ps.of_q, ps.first_k(part, p.parts), gk, dgk);
    }
    // over the heads of the wave, then over the waves, in a fixed order
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int o = GL; o < 64; o <<= 1) {
            dgq[i] += __shfl_xor(dgq[i], o);
            dgk[i] += __shfl_xor(dgk[i], o);
        }
        if (ln.slot == 0) {
            red[w][0][8 * ln.j + i] = dgq[i];
            red[w][1][8 * ln.j + i] = dgk[i];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.D; i += 64 * WAVES) {
        const int t = i >= p.D, d = i - t * p.D;
        float sum = red[0][t][d];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += red[v][t][d];
        p.part[(int64_t)blockIdx.x * 2 * p.D + i] = sum;
    }
}

// dgamma (+)= the sum over the workgroups' planes: a wave for four columns, all loads under way together.
__global__ void __launch_bounds__(64) rope_finalize_kernel(RopeFinalizeArgs p) {
    const int l = threadIdx.x, c = blockIdx.x * 4;
    f32x4 v[kRopeBlocks / 64];
#pragma unroll
    for (int i = 0; i < kRopeBlocks / 64; ++i) {
        v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (l + 64 * i < p.blocks) v[i] = *(const f32x4*)(p.part + (int64_t)(l + 64 * i) * 2 * p.D + c);
    }
#pragma unroll
    for (int i = 1; i < kRopeBlocks / 64; ++i) v[0] += v[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[0][e] += __shfl_xor(v[0][e], o);
    if (l) return;
    float* out = c < p.D ? p.dgamma_q + c : p.dgamma_k + c - p.D;
    if (p.accumulate) v[0] += *(const f32x4*)out;
    *(f32x4*)out = v[0];
}

// Parts of a row: more than one while there are fewer rows than 16 waves to a compute unit.  Backward, whose waves go on to further rows: about
// four passes to a part, so that the waves end together, and an odd number, so that a wave doesn't meet the same part in every row. us, parts 1 / 2 /
// 3 / 4 / 5 / 6: 5003 rows of 64 + 8 heads (18 passes) 70.6 / 64.5 / 63.9 / 65.3 / 62.3 / 62.0; 8192 rows of 32 + 8 (10) 61.8 / 60.1 / 59.4 / 61.9 / 59.4 / 61.1;
// 5003 of 8 + 2, D = 256 (5) 26.0 / 29.9 / 30.4 / 39.5.  (Forward, 8192 rows of 32 + 8: 39.3 / 45.5, each part forms the row's factors anew.)
template <int GL>
static int rope_parts(int64_t M, int H, int G, bool backward) {
    const int all = RopePasses<GL>(H, G).all;
    const int64_t want = std::max((16 * kComputeUnits + M - 1) / std::max<int64_t>(M, 1), (int64_t)(backward ? (all + 2) / 4 | 1 : 1));
    return (int)std::min<int64_t>(want, all);
}
template <class F>
static auto with_lanes(int D, F&& f) {
    if (D <= 64) return f(std::integral_constant<int, 8>{});
    if (D <= 128) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, 32>{});
}

template <class F>
static hipError_t with_pairs(bool interleaved, F&& f) { return interleaved ? f(std::true_type{}) : f(std::false_type{}); }

hipError_t launch_rope_fwd(RopeArgs a, bool interleaved, hipStream_t st) {
    return with_lanes(a.D, [&](auto gl) {
        a.parts = rope_parts<gl()>(a.M, a.H, a.G, false);
        return with_pairs(interleaved, [&](auto inter) {
            // (a launch has fewer than 2^32 threads: 64 a row)
            constexpr int64_t ROWS = 1 << 25;
            hipError_t e = hipSuccess;
            for (int64_t left = a.M; left > 0 && e == hipSuccess; left -= ROWS) {
                a.M = std::min(left, ROWS);
                const int64_t blocks = (a.M * a.parts + kRopeThreads / 64 - 1) / (kRopeThreads / 64);
                hipLaunchKernelGGL((rope_fwd_kernel<gl(), inter()>), dim3((unsigned)blocks), dim3(kRopeThreads), 0, st, a);
                e = hipGetLastError();
                a.q += a.M * a.ldq;
                a.k += a.M * a.ldk;
                a.q_out += a.M * a.ldqo;
                a.k_out += a.M * a.ldko;
                a.pos += a.M;
            }
            return e;
        });
    });
}

int rope_blocks(int64_t M, int H, int G, int D) {
    return with_lanes(D, [&](auto gl) {
        const int64_t n = (M * rope_parts<gl()>(M, H, G, true) + rope_bwd_waves(gl()) - 1) / rope_bwd_waves(gl());
        return (int)(n < kRopeBlocks ? n : kRopeBlocks);
    });
}

hipError_t launch_rope_bwd(RopeArgs a, bool interleaved, const RopeFinalizeArgs& f, hipStream_t st) {
    if (f.blocks > 0) {
        const hipError_t e = with_lanes(a.D, [&](auto gl) {
            a.parts = rope_parts<gl()>(a.M, a.H, a.G, true);
            return with_pairs(interleaved, [&](auto inter) {
                hipLaunchKernelGGL((rope_bwd_kernel<gl(), inter()>), dim3(f.blocks), dim3(64 * rope_bwd_waves(gl())), 0, st, a);
                return hipGetLastError();
            });
        });
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(rope_finalize_kernel, dim3(2 * a.D / 4), dim3(64), 0, st, f);
    return hipGetLastError();
}

}  // namespace lf
