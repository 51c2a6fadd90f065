// The LoRA linear layer for many requests at once: every row names its adapter, or none, in an array on the device.
//     S[i] = s_g X[i] A_g^T        this file        (bf16, columns past the adapter's rank zero)
//     Y[i] = X[i] W^T + S[i] B_g^T  lf_gemm_ring.hip (the small GEMM tiles; the second term on the accumulators: request_term)
// The first is bound by the latency of ids, ranks and adapters, one after the other, and by the reading of the adapters: a wave takes two columns of the
// rank for one row, so that a decode step of a few rows is spread over the chip, or, where many rows come as chunks of few requests, 16 rows
// go through MFMAs at once.  Two launches: with S formed in the tiles of the second product every column tile would form it again.
#include <algorithm>

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

// Columns of the rank to a wave.  us, whole layer, 4 / 2 / 1: 64 rows, K = 4096, r = 16 17.6 / 17.1 / 16.9; 32 rows, K = 14336 50.3 / 46.3 / 45.8; 200 rows, r = 64
// 101.1 / 99.8 / 101.0; 2048 rows, 37 single ones among them, r = 32 74.0 / 72.5 / 74.9.
constexpr int kDownColumns = 2;

// Columns j0, j0 + 1 of one row of S, by a wave.
__device__ __forceinline__ void request_row(const RequestDownArgs& p, int row, int j0) {
    constexpr int J = kDownColumns;
    const int l = threadIdx.x & 63;
    int id = p.ids[row];
    if (id >= p.P) id = -1;
    const int rank = id < 0 ? 0 : p.ranks ? min(p.ranks[id], p.r) : p.r;
    float v[J] = {};
    if (rank > j0) {
        const lora_bf16* x = p.X + (int64_t)row * p.K;
        const lora_bf16* a = p.A + ((int64_t)id * p.r + j0) * p.K;
#pragma unroll 4
        for (int k = 8 * l; k < p.K; k += 512) {
            const u32x4 xk = *(const u32x4*)(x + k);
#pragma unroll
            for (int j = 0; j < J; ++j) v[j] = dot8(xk, *(const u32x4*)(a + (int64_t)j * p.K + k), v[j]);
        }
        const float s = p.s[id];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            v[j] = sum_of_wave(v[j]);
            v[j] = j0 + j < rank ? s * v[j] : 0.f;                 // (padding of A may hold anything)
        }
    }
    if (l == 0) *(uint32_t*)(p.S + (int64_t)row * p.r + j0) = pack_bf16x2(v[0], v[1]);
}

__global__ void __launch_bounds__(64) request_rows_kernel(RequestDownArgs p) { request_row(p, blockIdx.x, blockIdx.y * kDownColumns); }

// Many rows: the 16-row tiles of one adapter by MFMAs, 16 columns of the rank to a workgroup, every eighth 64-deep slab of the contraction to a
// wave, four of them under way at once (a lane's two 16-byte loads of a row's slab lie side by side).  The rows of the other tiles go to
// further workgroups of the launch, a wave for each row and two columns, which find nothing to do where the tile is of one adapter.
// (One after the other in their own workgroups the adapters of such tiles, 37 requests of one token among 2048 rows, took 57 us.)
constexpr int kTileWaves = 8;
struct RequestTileArgs { RequestDownArgs d; int tiles, parts; };       // parts: of the rank, 16 columns each
__global__ void __launch_bounds__(64 * kTileWaves) request_tile_kernel(RequestTileArgs a) {
    __shared__ f32x4 red[kTileWaves][64];
    const RequestDownArgs& p = a.d;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool by_rows = (int)blockIdx.x >= a.tiles * a.parts;
    // by rows: PER waves to a row for each part
    constexpr int PER = 16 / kDownColumns;
    const int unit = by_rows ? ((int)blockIdx.x - a.tiles * a.parts) * kTileWaves + w : 0;
    const int own = unit / (PER * a.parts), row0 = by_rows ? own & ~15 : (int)blockIdx.x / a.parts * 16;
    if (row0 >= p.M) return;
    const int row = row0 + (l & 15);
    int id = p.ids[min(row, p.M - 1)];
    if (id < 0 || id >= p.P) id = -1;
    const int g = __builtin_amdgcn_readfirstlane(id);
    const bool one = __all(id == g);
    if (by_rows) {
        if (!one && own < p.M) request_row(p, own, unit % (PER * a.parts) * kDownColumns);
        return;
    }
    if (!one) return;
    const int j0 = (int)blockIdx.x % a.parts * 16, rank = g < 0 ? 0 : p.ranks ? min(p.ranks[g], p.r) : p.r;
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
    if (rank > j0) {
        const lora_bf16* x = p.X + (int64_t)min(row, p.M - 1) * p.K + 16 * (l >> 4);
        const lora_bf16* ag = p.A + ((int64_t)g * p.r + j0 + (l & 15)) * p.K + 16 * (l >> 4);
        constexpr int U = 4;
        for (int k = 64 * w; k < p.K; k += 64 * kTileWaves * U) {
            bf16x8 xf[U][2], af[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = min(k + 64 * kTileWaves * u, p.K - 64) + 8 * h;       // (past the end: brought, not used)
                    xf[u][h] = __builtin_bit_cast(bf16x8, *(const u32x4*)(x + at));
                    af[u][h] = __builtin_bit_cast(bf16x8, *(const u32x4*)(ag + at));
                }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + 64 * kTileWaves * u < p.K)
#pragma unroll
                    for (int h = 0; h < 2; ++h) acc = LF_MFMA(af[u][h], xf[u][h], acc);
        }
    }
    red[w][l] = acc;
    __syncthreads();
    if (w || row >= p.M) return;
#pragma unroll
    for (int i = 1; i < kTileWaves; ++i) acc += red[i][l];
    const int c = j0 + 4 * (l >> 4);
    const float s = g < 0 ? 0.f : p.s[g];
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = c + e < rank ? s * acc[e] : 0.f;
    *(u32x2*)(p.S + (int64_t)row * p.r + c) = u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
}

// Waves for single rows up to 512 of them (r = 64: 256), whatever adapters they have, in workgroups of their own, which start sooner than those of eight waves: us, rows /
// tiles, with four columns to a wave: 3 rows, K = 1024 2.7 / 3.4; 64 rows of 48 adapters, K = 4096, r = 16 4.0 / 6.2; 200 rows of 106 adapters, r = 64 13.8 / 16.5.
// (Whole layer, 4096 -> 4096, one adapter: 128 rows, r = 16 15.5 / 21.6; 512 rows 28.0 / 31.7; r = 64, 256 rows 25.4 / 26.2, 512 rows 38.4 / 33.5; an adapter for
// each row: level.)  With two: 2.7, 3.9, 12.4 (27 MB, 2.2 TB/s); 2048 rows on tiles 12.4 (17 MB of X).
static hipError_t launch_request_down(const RequestDownArgs& a, hipStream_t st) {
    if (a.M <= 512 && a.M * a.r <= 512 * 32) {
        hipLaunchKernelGGL(request_rows_kernel, dim3((unsigned)a.M, (unsigned)a.r / kDownColumns), dim3(64), 0, st, a);
        return hipGetLastError();
    }
    // Rows of a launch: a launch has fewer than 2^32 threads, and these are up to 2176 a row (r = 64).
    constexpr int kRows = 1 << 20;
    static_assert((64ll * kTileWaves * (kRows / 16 * 4 + (int64_t)kRows * (16 / kDownColumns) * 4 / kTileWaves)) < 1ll << 32, "threads of a launch");
    for (int64_t row = 0; row < a.M; row += kRows) {
        const int rows = (int)std::min<int64_t>(a.M - row, kRows);
        const RequestTileArgs t{{a.X + row * a.K, a.A, a.ids + row, a.ranks, a.s, a.S + row * a.r, rows, a.K, a.r, a.P}, (rows + 15) / 16, a.r / 16};
        const int64_t by_rows = ((int64_t)rows * (16 / kDownColumns) * t.parts + kTileWaves - 1) / kTileWaves;
        hipLaunchKernelGGL(request_tile_kernel, dim3((unsigned)((int64_t)t.tiles * t.parts + by_rows)), dim3(64 * kTileWaves), 0, st, t);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
