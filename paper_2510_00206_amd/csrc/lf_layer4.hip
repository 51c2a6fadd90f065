// The LoRA linear layer for many requests over 4-bit weights:
//     S[i] = s_g X[i] A_g^T             lf_requests.hip
//     Y[i] = X[i] W^T + S[i] B_g^T,     W[n,k] = e2m1(codes[n,k]) 2^(exps[n,k/32] - 127)
// The codes are widened to bf16 (exact, one instruction for two) on their way into the matrix instructions, so that no product is rounded and the sums
// are those of bf16 weights.  A lane takes 16 bytes of a row of codes: 32 entries, which share one power of two.  Its 16-byte load is four matrix steps, for
// which the contraction is numbered as the lanes hold it: step j of a block of 128 has entries 32 q + 8 j .. + 7 in the lanes with l >> 4 = q, of X as of W.
#include <algorithm>

#include "lf_gemm_parts.h"
#include "lf_gemm_ring.h"
#include "lf_request_term.h"
#include "lf_serve.h"

namespace lf {

struct LayerArgs {
    RingRequestArgs t;                 // tok X, ltok S, lout B, res Y
    const uint8_t* codes; const uint8_t* exps;
};

// Few rows: bound by the reading of the weights.  A workgroup has NI x 16 columns and MI x 16 rows, its NW waves every NW-th block of 128 of the contraction; the
// adapters' term is formed by waves of its own, 16 rows to each, beside them.  Sums of the waves are added in LDS in a fixed order.
template <int MI_, int NI_, int NW_>
struct FewLayer {
    static constexpr int MI = MI_, NI = NI_, NW = NW_, TM = 16 * MI, TN = 16 * NI;
    struct Term {                      // of one wave
        static constexpr int MI = 1, NI = NI_, NW = NW_, CW = MI_, LDS = 160 * 1024, TN = 16 * NI_, SUBS = 0;
        static constexpr bool AHEAD = false;
    };
    static constexpr int SUMS = (NW + 1) * MI * NI * 1024, LDS = SUMS + MI * (int)sizeof(RequestList<Term>);
    static_assert(LDS <= 160 * 1024, "a compute unit's LDS");
};

template <class C>
__global__ void __launch_bounds__(64 * (C::NW + C::MI)) layer_few_kernel(LayerArgs p) {
    constexpr int MI = C::MI, NI = C::NI, NW = C::NW;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;
    const int tn = (int)blockIdx.x % p.t.tiles_n, tm = (int)blockIdx.x / p.t.tiles_n;
    const int c0 = tn * C::TN, K = p.t.KC;
    RowTile rt{};
    rt.row_start = p.t.row_lo + tm * C::TM;
    rt.rows = min(C::TM, p.t.row_hi - rt.row_start);
    f32x4* sums = (f32x4*)smem;                                // [wave, the term last][mi][ni][lane]
    if (w >= NW) {
        if (p.t.P > 0) {
            using T = typename C::Term;
            const int mi = w - NW;
            f32x4 acc[1][NI];
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[0][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (16 * mi < rt.rows) {
                RequestTerm<T> term(p.t, rt, c0, mi, 0, ((RequestList<T>*)(smem + C::SUMS))[mi]);
                term.form(acc);
            }
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) sums[((NW * MI + mi) * NI + ni) * 64 + l] = acc[0][ni];
        }
    } else {
        f32x4 acc[MI][NI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
        const lora_bf16* x[MI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) x[mi] = p.t.tok + (int64_t)(rt.row_start + min(16 * mi + c, rt.rows - 1)) * K;
        const uint8_t* codes = p.codes + (int64_t)(c0 + c) * (K / 2);
        const uint8_t* exps = p.exps + (int64_t)(c0 + c) * (K / 32);
        const int blocks = (K + 127) / 128;
        for (int b = w; b < blocks; b += NW) {
            const bool in = 128 * b + 32 * q < K;              // (the last block may be half a one)
            const int k = in ? 128 * b + 32 * q : 128 * b;
            u32x4 code[NI], xr[MI][4];
            float scale[NI];
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                code[ni] = *(const u32x4*)(codes + (int64_t)ni * 16 * (K / 2) + k / 2);
                scale[ni] = exp2_of_biased(exps[(int64_t)ni * 16 * (K / 32) + k / 32]);
            }
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int j = 0; j < 4; ++j) xr[mi][j] = *(const u32x4*)(x[mi] + k + 8 * j);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) {
                    bf16x8 wf = from_fp4(code[ni][j], scale[ni]);
                    if (!in) wf = bf16x8{};
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) {
                        const bf16x8 xf = in ? __builtin_bit_cast(bf16x8, xr[mi][j]) : bf16x8{};
                        acc[mi][ni] = LF_MFMA(wf, xf, acc[mi][ni]);
                    }
                }
        }
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) sums[((w * MI + mi) * NI + ni) * 64 + l] = acc[mi][ni];
    }
    __syncthreads();
    const int parts = p.t.P > 0 ? NW + 1 : NW;
    for (int b = w; b < MI * NI; b += NW + MI) {
        const int mi = b / NI, ni = b % NI, row = 16 * mi + c;
        f32x4 y = sums[b * 64 + l];
        for (int i = 1; i < parts; ++i) y += sums[(i * MI * NI + b) * 64 + l];
        if (row < rt.rows)
            *(u32x2*)(p.t.res + (int64_t)(rt.row_start + row) * p.t.NC + c0 + 16 * ni + 4 * q) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
    }
}

template <class C>
static hipError_t launch_few(LayerArgs a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};       // one per instantiation
    hipError_t e = allow_lds((const void*)layer_few_kernel<C>, C::LDS, allowed);
    a.t.tiles_n = a.t.NC / C::TN;
    // (a launch has fewer than 2^32 threads)
    const int rows = (int)std::min<int64_t>((1ll << 31) / (64 * (C::NW + C::MI)) / a.t.tiles_n, 1 << 20) * C::TM;
    for (int row = 0; row < a.t.M && e == hipSuccess; row += rows) {
        a.t.row_lo = row;
        a.t.row_hi = std::min(a.t.M, row + rows);
        a.t.tiles_m = (a.t.row_hi - row + C::TM - 1) / C::TM;
        hipLaunchKernelGGL(layer_few_kernel<C>, dim3((unsigned)((int64_t)a.t.tiles_m * a.t.tiles_n)), dim3(64 * (C::NW + C::MI)), C::LDS, st, a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_quantised_requests(const QuantisedRequestArgs& a, hipStream_t st) {
    hipError_t e = a.r.P > 0 ? launch_request_down(a.r, st) : hipSuccess;
    if (e != hipSuccess) return e;
    LayerArgs g{};
    g.t.tok = a.r.X;
    g.t.ltok = a.r.S;
    g.t.lout = a.r.B;
    g.t.res = a.r.Y;
    g.t.M = a.r.M;
    g.t.KC = a.r.K;
    g.t.NC = a.r.N;
    g.t.ids = a.r.ids;
    g.t.ranks = a.r.ranks;
    g.t.lr = a.r.r;
    g.t.P = a.r.P;
    g.codes = a.codes;
    g.exps = a.exps;
    if (a.r.M <= 16) return launch_few<FewLayer<1, 1, 8>>(g, st);
    if (a.r.M <= 32) return launch_few<FewLayer<2, 2, 8>>(g, st);
    return launch_few<FewLayer<4, 2, 8>>(g, st);
}

}  // namespace lf
