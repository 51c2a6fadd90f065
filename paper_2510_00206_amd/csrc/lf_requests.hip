// The LoRA linear layer for many requests at once: every row names its adapter, or none, in an array on the device.
//     S[i] = s_g X[i] A_g^T        this file        (bf16, columns past the adapter's rank zero)
//     Y[i] = X[i] W^T + S[i] B_g^T  lf_gemm_ring.hip (the small GEMM tiles; the second term on the accumulators: request_term)
// The first is bound by the reading of the adapters: up to a few hundred rows, which may all have adapters of their own, a wave takes four
// columns of the rank for one row or for four rows, which share what they read of A if they share the adapter.  More rows come as
// chunks of few requests: 16 rows to a workgroup by MFMAs, once for every adapter among them.
#include "lf_gemm_parts.h"
#include "lf_gemm_ring.h"
#include "lf_serve.h"

namespace lf {

struct RequestDownArgs {
    const lora_bf16* X; const lora_bf16* A; const int32_t* ids; const int32_t* ranks; const float* s; lora_bf16* S;
    int M, K, r, P;
};

__device__ __forceinline__ float dot8(u32x4 a, u32x4 b, float c) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = a[i], y = b[i];
        c = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), c, false);
    }
    return c;
}

__device__ __forceinline__ float sum_of_wave(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

constexpr int kDownColumns = 4;                    // columns of the rank to a wave

template <int ROWS>
__global__ void __launch_bounds__(64) request_rows_kernel(RequestDownArgs p) {
    constexpr int J = kDownColumns;
    const int l = threadIdx.x, row0 = blockIdx.x * ROWS, j0 = blockIdx.y * J;
    int id[ROWS], rank[ROWS];
    bool shared = true;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        id[i] = row0 + i < p.M ? p.ids[row0 + i] : -1;
        if (id[i] >= p.P) id[i] = -1;
        rank[i] = id[i] < 0 ? 0 : p.ranks ? min(p.ranks[id[i]], p.r) : p.r;
        shared = shared && id[i] == id[0];
    }
    float acc[ROWS][J];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = 0.f;
    const u32x4 zero{0u, 0u, 0u, 0u};
    auto x_at = [&](int i, int k) { return *(const u32x4*)(p.X + (int64_t)(row0 + i) * p.K + k); };
    auto a_at = [&](int i, int j, int k) { return *(const u32x4*)(p.A + ((int64_t)id[i] * p.r + j0 + j) * p.K + k); };
    if (shared) {
        if (rank[0] > j0) {
#pragma unroll 2
            for (int k = 8 * l; k < p.K; k += 512) {
                u32x4 x[ROWS], a[J];
#pragma unroll
                for (int i = 0; i < ROWS; ++i) x[i] = row0 + i < p.M ? x_at(i, k) : zero;
#pragma unroll
                for (int j = 0; j < J; ++j) a[j] = a_at(0, j, k);
#pragma unroll
                for (int i = 0; i < ROWS; ++i)
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[i][j] = dot8(x[i], a[j], acc[i][j]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            if (rank[i] <= j0) continue;
#pragma unroll 4
            for (int k = 8 * l; k < p.K; k += 512) {
                const u32x4 x = x_at(i, k);
#pragma unroll
                for (int j = 0; j < J; ++j) acc[i][j] = dot8(x, a_at(i, j, k), acc[i][j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (row0 + i >= p.M) break;
        const float s = id[i] < 0 ? 0.f : p.s[id[i]];
        float v[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            v[j] = sum_of_wave(acc[i][j]);
            v[j] = j0 + j < rank[i] ? s * v[j] : 0.f;              // (padding of A may hold anything)
        }
        if (l == 0) *(u32x2*)(p.S + (int64_t)(row0 + i) * p.r + j0) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
}

// 16 rows by 16 columns of the rank to a workgroup, every eighth 64-deep slab of the contraction to a wave, four of them under way at
// once; a lane's two 16-byte loads of a row's slab lie side by side.
constexpr int kTileWaves = 8;
__global__ void __launch_bounds__(64 * kTileWaves) request_tile_kernel(RequestDownArgs p) {
    __shared__ f32x4 red[kTileWaves][64];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = blockIdx.x * 16 + (l & 15), j0 = blockIdx.y * 16;
    int id = row < p.M ? p.ids[row] : -1;
    if (id >= p.P) id = -1;
    const lora_bf16* x = p.X + (int64_t)min(row, p.M - 1) * p.K + 16 * (l >> 4);
    f32x4 all = f32x4{0.f, 0.f, 0.f, 0.f};
    uint32_t todo = (uint32_t)__ballot(id >= 0) & 0xFFFFu;
    while (todo) {
        const int g = __builtin_amdgcn_readlane(id, __builtin_ctz(todo));
        todo &= ~(uint32_t)__ballot(id == g);
        if (p.ranks && p.ranks[g] <= j0) continue;
        const lora_bf16* a = p.A + ((int64_t)g * p.r + j0 + (l & 15)) * p.K + 16 * (l >> 4);
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int U = 4;
        for (int k = 64 * w; k < p.K; k += 64 * kTileWaves * U) {
            bf16x8 xf[U][2], af[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = min(k + 64 * kTileWaves * u, p.K - 64) + 8 * h;       // (past the end: brought, not used)
                    xf[u][h] = __builtin_bit_cast(bf16x8, *(const u32x4*)(x + at));
                    af[u][h] = __builtin_bit_cast(bf16x8, *(const u32x4*)(a + at));
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + 64 * kTileWaves * u < p.K)
#pragma unroll
                    for (int h = 0; h < 2; ++h) acc = LF_MFMA(af[u][h], xf[u][h], acc);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) all[e] = id == g ? acc[e] : all[e];
    }
    red[w][l] = all;
    __syncthreads();
    if (w || row >= p.M) return;
#pragma unroll
    for (int i = 1; i < kTileWaves; ++i) all += red[i][l];
    const int c = j0 + 4 * (l >> 4), rank = id < 0 ? 0 : p.ranks ? p.ranks[id] : p.r;
    const float s = id < 0 ? 0.f : p.s[id];
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = c + e < rank ? s * all[e] : 0.f;
    *(u32x2*)(p.S + (int64_t)row * p.r + c) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
}

static hipError_t launch_request_down(const RequestDownArgs& a, hipStream_t st) {
    const unsigned parts = (unsigned)a.r / kDownColumns;
    if (a.M <= 128) {
        hipLaunchKernelGGL(request_rows_kernel<1>, dim3((unsigned)a.M, parts), dim3(64), 0, st, a);
    } else if (a.M <= 512) {
        hipLaunchKernelGGL(request_rows_kernel<4>, dim3((unsigned)(a.M + 3) / 4, parts), dim3(64), 0, st, a);
    } else {
        hipLaunchKernelGGL(request_tile_kernel, dim3((unsigned)(a.M + 15) / 16, (unsigned)a.r / 16), dim3(64 * kTileWaves), 0, st, a);
    }
    return hipGetLastError();
}

hipError_t launch_requests(const RequestArgs& a, hipStream_t st) {
    hipError_t e = launch_request_down(RequestDownArgs{a.X, a.A, a.ids, a.ranks, a.s, a.S, a.M, a.K, a.r, a.P}, st);
    RingPart part[2];
    const int n = plan_ring(a.M, a.K, a.N, part);
    for (int i = 0; i < n && e == hipSuccess; ++i) {
        RingRequestArgs g{a.X, a.W, a.S, a.B, a.Y, a.M, a.K, a.N, 0, part[i].tiles_m, part[i].tiles_n, part[i].row_lo, part[i].row_hi, a.ids, a.ranks, a.r, a.P, {}};
        g.tb.G = 1;
        g.tb.row0[1] = a.M;
        e = launch_ring_requests(part[i].kind, g, st);
    }
    return e;
}

}  // namespace lf
