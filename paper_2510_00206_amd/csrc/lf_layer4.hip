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

constexpr int kBlock = 128;            // of the contraction, the last one may be half of it

struct LayerArgs {
    RingRequestArgs t;                 // tok X, ltok S, lout B, res Y
    const uint8_t* codes; const uint8_t* exps;
};

// A lane's 32 codes and their power of two: row n of W, entries k .. k + 31.
__device__ __forceinline__ void load_codes(const LayerArgs& p, int n, int k, u32x4& code, uint32_t& e) {
    code = *(const u32x4*)(p.codes + (int64_t)n * (p.t.KC / 2) + k / 2);
    e = p.exps[(int64_t)n * (p.t.KC / 32) + k / 32];
}

// A lane's place in the contraction: entries 32 q .. of a block; in the half block at the end, if there is one, 16 q + 8 j .. of two steps, of which its load
// holds one half.
__device__ __forceinline__ int entry_of(int b, int whole, int q) { return kBlock * b + (b < whole ? 32 * q : 32 * (q >> 1)); }

// A matrix instruction from assembly with the accumulator tied in place (the compiler's own moved accumulators between registers).  FROM_VALU: its operands may come
// straight from the vector ALU, which takes two wait states.
template <bool FROM_VALU>
__device__ __forceinline__ void mfma_in_place(f32x4& acc, bf16x8 a, bf16x8 b) {
    if constexpr (FROM_VALU) asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
    else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(a), "v"(b));
}

// Four bytes to a lane, to M0 (as the copy before it left it) + IMM + 4 * lane.
template <int IMM>
__device__ __forceinline__ void copy4_to_lds(const char* biased_base, uint32_t lane_byte_off) {
    asm volatile("global_load_lds_dword %0, %1 offset:%2" :: "v"(lane_byte_off), "s"(biased_base), "n"(IMM) : "memory");
}

// ---- few rows ---------------------------------------------------------------------------------------
// Bound by the reading of the weights.  A workgroup has NI x 16 columns and MI x 16 rows, its NW waves every NW-th block of the contraction, U blocks under way
// at once; the adapters' term is formed by TW waves of its own beside them, which share its steps.  Sums of the waves are added in LDS in a fixed order.
template <int MI_, int NI_, int NW_, int TW_, int U_>
struct FewLayer {
    static constexpr int MI = MI_, NI = NI_, NW = NW_, TW = TW_, U = U_, TM = 16 * MI, TN = 16 * NI;
    struct Term {                      // of one wave
        static constexpr int MI = MI_, NI = NI_, NW = NW_, CW = TW_, LDS = 160 * 1024, TN = 16 * NI_, SUBS = 0, EVERY = TW_, HELD = 0;
        static constexpr bool AHEAD = false;
    };
    static constexpr int SUMS = (NW + TW) * MI * NI * 1024, LDS = SUMS + TW * (int)sizeof(RequestList<Term>);
    static_assert(LDS <= 160 * 1024, "a compute unit's LDS");
};

template <class C, bool TERM>
__global__ void __launch_bounds__(64 * (C::NW + (TERM ? C::TW : 0))) layer_few_kernel(LayerArgs p) {
    constexpr int MI = C::MI, NI = C::NI, NW = C::NW, U = C::U, WAVES = NW + (TERM ? C::TW : 0);
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;
    const int tn = (int)blockIdx.x % p.t.tiles_n, tm = (int)blockIdx.x / p.t.tiles_n;
    const int c0 = tn * C::TN, K = p.t.KC;
    RowTile rt{};
    rt.row_start = p.t.row_lo + tm * C::TM;
    rt.rows = min(C::TM, p.t.row_hi - rt.row_start);
    f32x4* sums = (f32x4*)smem;                                // [wave][mi][ni][lane]
    f32x4 acc[MI][NI];
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (TERM && w >= NW) {
        using T = typename C::Term;
        RequestTerm<T> term(p.t, rt, c0, 0, 0, ((RequestList<T>*)(smem + C::SUMS))[w - NW], w - NW);
        term.form(acc);
    } else {
        const lora_bf16* x[MI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) x[mi] = p.t.tok + (int64_t)(rt.row_start + min(16 * mi + c, rt.rows - 1)) * K;
        const int whole = K / kBlock, blocks = (K + kBlock - 1) / kBlock;
        for (int b0 = w; b0 < blocks; b0 += NW * U) {
            u32x4 code[U][NI], xr[U][MI][4];
            uint32_t e[U][NI];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int b = min(b0 + NW * u, blocks - 1), k = entry_of(b, whole, q), kx = b < whole ? k : kBlock * b + 16 * q;
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) load_codes(p, c0 + 16 * ni + c, k, code[u][ni], e[u][ni]);
#pragma unroll
                for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                    for (int j = 0; j < 4; ++j) xr[u][mi][j] = *(const u32x4*)(x[mi] + kx + (b < whole ? 8 * j : 8 * (j & 1)));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int b = b0 + NW * u;
                if (b >= blocks) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j == 2 && b >= whole) break;
#pragma unroll
                    for (int ni = 0; ni < NI; ++ni) {
                        const uint32_t half = q & 1 ? code[u][ni][2 + (j & 1)] : code[u][ni][j & 1];
                        const bf16x8 wf = from_fp4(b < whole ? code[u][ni][j] : half, exp2_of_biased(e[u][ni]));
#pragma unroll
                        for (int mi = 0; mi < MI; ++mi) acc[mi][ni] = LF_MFMA(wf, __builtin_bit_cast(bf16x8, xr[u][mi][j]), acc[mi][ni]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) sums[((w * MI + mi) * NI + ni) * 64 + l] = acc[mi][ni];
    __syncthreads();
    for (int b = w; b < MI * NI; b += WAVES) {
        const int mi = b / NI, ni = b % NI, row = 16 * mi + c;
        f32x4 y = sums[b * 64 + l];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) y += sums[(i * MI * NI + b) * 64 + l];
        if (row < rt.rows)
            *(u32x2*)(p.t.res + (int64_t)(rt.row_start + row) * p.t.NC + c0 + 16 * ni + 4 * q) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
    }
}

// ---- more rows --------------------------------------------------------------------------------------
// X, the codes and the exponents go through a ring of NS blocks in LDS, filled by CW waves that do nothing else.  A wave's 16 MI x 16 NI tile is one stream of
// instructions over the blocks: a matrix instruction to a slot, and between them the reads of the fragments of X, three ahead of their use, and the widening of the next
// step's codes.  (Codes straight from memory into the registers of the lanes that use them, 16 bytes of a row to each: neighbouring lanes have other rows, so that a
// load takes 64 cycles of the address unit instead of 16, and one of exponents, a byte to a lane, as many; 2048 rows, 4096 -> 4096: 71 us, 1.9 us a block.)
template <int MI_, int NI_, int WM_, int WN_, int NS_, int CW_>
struct RingLayer {
    static constexpr int MI = MI_, NI = NI_, WM = WM_, WN = WN_, NS = NS_, CW = CW_, NW = WM * WN, THREADS = 64 * NW;
    static constexpr int TM = 16 * MI * WM, TN = 16 * NI * WN;
    // a block: X, then of every copying wave the codes of RW rows, their exponents (four bytes a row, for 64 rows), and the four bytes behind those
    static constexpr int XB = TM * 2 * kBlock, RW = TN / CW, PART = RW * (kBlock / 2) + 512, STAGE = XB + CW * PART;
    static constexpr int XC = XB / 1024 / CW, CC = RW / 16;                         // copies of a wave: of X, of codes (of exponents: one or two)
    static constexpr int OUT = TM * TN * 2;
    static constexpr int HALVES = (MI + 3) / 4;                                     // the term is formed for 64 rows of a wave at a time
    struct Term {
        static constexpr int MI = MI_ > 4 ? MI_ / 2 : MI_, NI = NI_, NW = WM_ * WN_, CW = CW_, LDS = NS_ * STAGE, TN = 16 * NI_ * WN_, SUBS = 2, EVERY = 1;
        static constexpr int HELD = (MI_ - MI) * NI * 4;                            // the other rows' accumulators
        static constexpr bool AHEAD = false;
    };
    static constexpr int RING = NS * STAGE > OUT ? NS * STAGE : OUT;
    static constexpr int LDS = RING + NW * (int)sizeof(RequestList<Term>);
    static_assert(XB % (1024 * CW) == 0 && XC <= 8 && RW % 16 == 0 && RW <= 64, "copies of a block: whole, in reach of the immediates");
    static_assert((XC + CC + 2) * (NS - 2) < 64, "... and of the wait counter");
    static_assert(NS >= 3 && LDS <= 160 * 1024, "a compute unit's LDS");
};
// Position of 16-byte chunk ch of a row: of X (256 bytes), where the 16 rows of a fragment need 16 positions; of codes (64 bytes), where four rows share 256 bytes.
__device__ __forceinline__ int x_chunk(int row, int ch) { return ch ^ (row & 15); }
__device__ __forceinline__ int code_chunk(int row, int ch) { return ch ^ (row >> 2 & 3); }

// The copying waves.  Block b + NS - 1 goes where block b - 1 was, which every wave has left when it comes to the barrier in block b; behind that barrier block
// b + 1 has landed.  Exponents: the aligned four bytes with the first of a row's block, and, where rows are not whole blocks (SPLIT), the four behind
// them, since every other row's block starts in the middle.
template <class C, int N, int I = 0>
__device__ __forceinline__ void copy_rows(const char* biased, const uint32_t (&off)[N], uint32_t to) {
    if constexpr (I < N) {
        copy16_to_lds<pass_imm(N, I), I == 0>(biased, off[I], to + N / 2 * 1024);
        copy_rows<C, N, I + 1>(biased, off, to);
    }
}
template <class C, bool SPLIT>
__device__ __forceinline__ void copying_wave(const LayerArgs& p, const RowTile& rt, int c0, int w, uint32_t lds) {
    constexpr int NS = C::NS, N = C::XC + C::CC + (SPLIT ? 2 : 1);
    const int l = threadIdx.x & 63, K = p.t.KC, whole = K / kBlock, blocks = (K + kBlock - 1) / kBlock;
    uint32_t xo[C::XC], co[C::CC], eo;
    auto form = [&](int bytes) {                               // valid bytes of a row of codes
#pragma unroll
        for (int i = 0; i < C::XC; ++i) {
            const int row = (w * C::XC + i) * 4 + l / 16, ch = min(x_chunk(row, l % 16), bytes / 4 - 1);
            xo[i] = ((uint32_t)min(row, rt.rows - 1) * (uint32_t)K + 8 * ch) * 2 + kCopyBias - pass_imm(C::XC, i);
        }
#pragma unroll
        for (int i = 0; i < C::CC; ++i) {
            const int row = w * C::RW + 16 * i + l / 4, ch = min(code_chunk(row, l % 4), bytes / 16 - 1);
            co[i] = (uint32_t)min(row, p.t.NC - 1 - c0) * (uint32_t)(K / 2) + 16 * ch + kCopyBias - pass_imm(C::CC, i);
        }
    };
    {
        // (M0 stands in the middle of the codes: the exponents' immediates count from there)
        constexpr int at = (C::CC - C::CC / 2) * 1024;
        eo = (uint32_t)min(w * C::RW + l % C::RW, p.t.NC - 1 - c0) * (uint32_t)(K / 32) + kCopyBias - at;
    }
    const char* x = (const char*)(p.t.tok + (int64_t)rt.row_start * K) - kCopyBias;
    const char* codes = (const char*)p.codes + (int64_t)c0 * (K / 2) - kCopyBias;
    const char* exps = (const char*)p.exps + (int64_t)c0 * (K / 32) - kCopyBias;
    // exponents to the array's end, from the tile's first row
    const uint32_t left = (uint32_t)min((int64_t)(p.t.NC - c0) * (K / 32), (int64_t)1 << 30);
    auto block = [&](int b, int stage) {
        if (b >= blocks) return;
        if (b >= whole) form(kBlock / 4);
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + stage * C::STAGE + w * C::XC * 1024);
        copy_rows<C, C::XC>(x + (int64_t)b * (2 * kBlock), xo, to);
        copy_rows<C, C::CC>(codes + (int64_t)b * (kBlock / 2), co, __builtin_amdgcn_readfirstlane(lds + stage * C::STAGE + C::XB + w * C::PART));
        constexpr int at = (C::CC - C::CC / 2) * 1024;
        const char* e = exps + (int64_t)b * (kBlock / 32);
        if constexpr (SPLIT) {
            // the offsets are even, from an array whose start is a multiple of 16, as is the tile's first row
            const uint32_t first = eo - (kCopyBias - at) + b * (kBlock / 32), down = first & 2u, behind = min(first - down + 4, left - 4);
            copy4_to_lds<at>(e, eo - down);
            copy4_to_lds<at + 256>(exps, behind + kCopyBias - at - 256);
        } else {
            copy4_to_lds<at>(e, eo);
        }
    };
    form(kBlock / 2);
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) block(s, s);
    if (blocks >= NS - 1) wait_slab_loads_but<N*(NS - 2)>();
    else wait_slab_loads();
    asm volatile("s_barrier" ::: "memory");
    int stage = NS - 1;
    for (int b = 0; b < whole; ++b) {
        if (b + NS - 1 <= blocks) wait_slab_loads_but<N*(NS - 3)>();
        else wait_slab_loads();
        asm volatile("s_barrier" ::: "memory");
        block(b + NS - 1, stage);
        stage = stage + 1 == NS ? 0 : stage + 1;
    }
}

template <class C, bool TERM>
__global__ void __launch_bounds__(C::THREADS + 64 * C::CW) layer_ring_kernel(LayerArgs p) {
    constexpr int MI = C::MI, NI = C::NI, NS = C::NS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    int tm, tn;
    tile_of_block(blockIdx.x, p.t.tiles_m, p.t.tiles_n, tm, tn);
    RowTile rt{};
    rt.row_start = p.t.row_lo + tm * C::TM;
    rt.rows = min(C::TM, p.t.row_hi - rt.row_start);
    const int c0 = tn * C::TN, K = p.t.KC, whole = K / kBlock, blocks = (K + kBlock - 1) / kBlock;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;
    if (w >= C::NW) {
        if (blocks > whole) copying_wave<C, true>(p, rt, c0, w - C::NW, lds_addr_of(smem));
        else copying_wave<C, false>(p, rt, c0, w - C::NW, lds_addr_of(smem));
    } else {
        const int wm = w % C::WM, wn = w / C::WM;
        f32x4 acc[MI][NI];
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (TERM) {
            using T = typename C::Term;
#pragma unroll
            for (int h = 0; h < C::HALVES; ++h) {
                RowTile half = rt;
                half.row_start += wm * 16 * MI + h * 64;
                half.rows = rt.rows - wm * 16 * MI - h * 64;
                if (half.rows <= 0) break;
                half.rows = min(half.rows, T::MI * 16);
                RequestTerm<T> term(p.t, half, c0, 0, wn, ((RequestList<T>*)(smem + C::RING))[w]);
                term.form(*(f32x4(*)[T::MI][NI]) & acc[h * 4]);
            }
        }
        asm volatile("s_barrier" ::: "memory");

        constexpr int FR = 4 * MI, SLOTS = FR * NI, STEP = MI * NI, AHEAD = 3;       // fragments of X and matrix instructions of a block; of a step
        // The next block's codes are asked for from slot HAND on, behind the barrier, and widened at the block's end.
        constexpr int WIDEN = SLOTS - STEP / 2, EARLY = WIDEN - 12 < 3 * STEP ? WIDEN - 12 : 3 * STEP, HAND = EARLY < 0 ? 0 : EARLY;
        static_assert(HAND <= (FR - AHEAD) * NI, "fragments of the next block are read behind the barrier");
        bf16x8 x[AHEAD + 1];
        u32x4 code[NI], coming[NI], wf[2][NI];
        uint32_t e[NI];
        float scale[NI];
        const int x0 = (wm * MI * 16 + c) * 256;
        // fragment f of a block: step f / MI, rows 16 (f % MI) ..
        auto read = [&](int stage, int f) {
            x[f % (AHEAD + 1)] = __builtin_bit_cast(bf16x8, *(const u32x4*)(smem + stage * C::STAGE + x0 + (f % MI) * 16 * 256 + (x_chunk(c, 4 * q + f / MI) << 4)));
        };
        // rows 16 nb .. of the tile (nb = wn * NI + ni): the part of their copying wave, and the row in it
        auto part_of = [&](int stage, int ni) { return smem + stage * C::STAGE + C::XB + (wn * NI + ni) / (C::RW / 16) * C::PART; };
        auto row_of = [&](int ni) { return (wn * NI + ni) % (C::RW / 16) * 16 + c; };
        const bool split = blocks > whole && (c & 1);           // this lane's rows' exponents start in the middle of four bytes
        auto read_codes = [&](int stage, int ni) {
            coming[ni] = *(const u32x4*)(part_of(stage, ni) + row_of(ni) * 64 + (code_chunk(c, q) << 4));
        };
        auto read_exp = [&](int stage, int ni) {
            const int byte = split ? (q < 2 ? 2 + q : 256 - 2 + q) : q;
            e[ni] = *(const uint8_t*)(part_of(stage, ni) + C::RW * 64 + row_of(ni) * 4 + byte);
        };
        auto arrive = [&](int ni) {
            code[ni] = coming[ni];
            scale[ni] = exp2_of_biased(e[ni]);
        };
        auto widen = [&](auto to, auto j, auto n) {            // two of the codes of step j: number n of 4 NI
            constexpr int ni = n() / 4, part = n() % 4;
            wf[to()][ni][part] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[ni][j()], scale[ni], part));
        };
        int stage = 0;
        // On the way into a block its first AHEAD fragments have been asked for, and the codes of its first step widened; the same is done for the next block.
        if (whole > 0) {
            auto zero = std::integral_constant<int, 0>{};
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                read_codes(0, ni);
                read_exp(0, ni);
                arrive(ni);
            }
            each<4 * NI>([&](auto n) { widen(zero, zero, n); });
#pragma unroll
            for (int f = 0; f < AHEAD; ++f) read(0, f);
        }
        for (int b = 0; b < whole; ++b) {
            const int next = stage + 1 == NS ? 0 : stage + 1;
            each<SLOTS>([&](auto slot) {
                constexpr int s = slot(), f = s / NI, ni = s % NI, j = s / STEP, in = s % STEP;
                if constexpr (s == HAND) asm volatile("s_barrier" ::: "memory");
                if constexpr (ni == 0) read(f + AHEAD < FR ? stage : next, (f + AHEAD) % FR);
                if constexpr (s >= HAND && s < HAND + NI) read_codes(next, s - HAND);
                if constexpr (s >= HAND + NI && s < HAND + 2 * NI) read_exp(next, s - HAND - NI);
                // (the next block's in the last half of a step; the others away from the step's last instruction, which the next one's first follows)
                constexpr int span = j == 3 ? STEP / 2 : STEP > 4 ? STEP - STEP / 4 : STEP, from = j == 3 ? STEP - span : 0;
                constexpr int v0 = slots_before(in - from, 4 * NI, span), v1 = slots_before(in + 1 - from, 4 * NI, span);
                each<v1 - v0>([&](auto k) {
                    constexpr int n = v0 + k();
                    if constexpr (j == 3 && n % 4 == 0) arrive(n / 4);
                    widen(std::integral_constant<int, (j + 1) & 1>{}, std::integral_constant<int, (j + 1) & 3>{}, std::integral_constant<int, n>{});
                });
                mfma_in_place<STEP <= 4 && in == 0>(acc[f % MI][ni], __builtin_bit_cast(bf16x8, wf[j & 1][ni]), x[f % (AHEAD + 1)]);
                __builtin_amdgcn_sched_barrier(0);
            });
            stage = next;
        }
        if (blocks > whole) {                                  // half a block, in two steps: 16 entries of each row to a lane
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const char* part = part_of(stage, ni);
                const u32x4 cd = *(const u32x4*)(part + row_of(ni) * 64 + (code_chunk(c, q >> 1) << 4));
                const float sc = exp2_of_biased(*(const uint8_t*)(part + C::RW * 64 + row_of(ni) * 4 + (split ? 2 : 0) + (q >> 1)));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 wh = from_fp4(q & 1 ? cd[2 + j] : cd[j], sc);
#pragma unroll
                    for (int mi = 0; mi < MI; ++mi) {
                        const bf16x8 xh = __builtin_bit_cast(bf16x8, *(const u32x4*)(smem + stage * C::STAGE + x0 + mi * 16 * 256 + (x_chunk(c, 2 * q + j) << 4)));
                        mfma_in_place<true>(acc[mi][ni], wh, xh);
                    }
                }
            }
        }
        ring_mfma_done<MI, NI>(acc);

        // way out: the bf16 tile through LDS, whole rows from there
        __syncthreads();
        constexpr int PITCH = C::TN * 2;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            const int r = (wm * MI + mi) * 16 + c;
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int slot = (wn * NI + ni) * 4 + q;
                *(u32x2*)(smem + r * PITCH + ((slot ^ ((r & 7) << 1)) << 3)) =
                    u32x2{pack_bf16x2(acc[mi][ni][0], acc[mi][ni][1]), pack_bf16x2(acc[mi][ni][2], acc[mi][ni][3])};
            }
        }
    }
    if (w >= C::NW) __syncthreads();
    __syncthreads();
    constexpr int CPR = C::TN / 8, ALL = C::THREADS + 64 * C::CW;
    lora_bf16* res = p.t.res + (int64_t)rt.row_start * p.t.NC + c0;
    const int cols = min(C::TN, p.t.NC - c0);
    for (int i = threadIdx.x; i < C::TM * CPR; i += ALL) {
        const int r = i / CPR, ch = i % CPR;
        if (r < rt.rows && ch * 8 < cols)
            __builtin_nontemporal_store(*(const u32x4*)(smem + r * (C::TN * 2) + ((ch ^ (r & 7)) << 4)), (u32x4*)(res + (int64_t)r * p.t.NC + ch * 8));
    }
}

// ---- launches ---------------------------------------------------------------------------------------
// f(kernel, first row, rows): launches of fewer than 2^32 threads.
template <class F>
static hipError_t by_rows(LayerArgs a, int tile_rows, int tile_columns, int threads, F&& f) {
    a.t.tiles_n = (a.t.NC + tile_columns - 1) / tile_columns;
    const int rows = (int)std::min<int64_t>((1ll << 31) / threads / a.t.tiles_n, 1 << 14) * tile_rows;
    hipError_t e = hipSuccess;
    for (int row = 0; row < a.t.M && e == hipSuccess; row += rows) {
        a.t.row_lo = row;
        a.t.row_hi = std::min(a.t.M, row + rows);
        a.t.tiles_m = (a.t.row_hi - row + tile_rows - 1) / tile_rows;
        e = f(a, dim3((unsigned)((int64_t)a.t.tiles_m * a.t.tiles_n)));
    }
    return e;
}

template <auto KERNEL>
static hipError_t launch_layer(const LayerArgs& a, int tile_rows, int tile_columns, int threads, int lds, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};       // one per kernel
    const hipError_t e = allow_lds((const void*)KERNEL, lds, allowed);
    if (e != hipSuccess) return e;
    return by_rows(a, tile_rows, tile_columns, threads, [&](const LayerArgs& b, dim3 grid) {
        hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, st, b);
        return hipGetLastError();
    });
}

template <class C>
static hipError_t launch_few(const LayerArgs& a, hipStream_t st) {
    if (a.t.P > 0) return launch_layer<layer_few_kernel<C, true>>(a, C::TM, C::TN, 64 * (C::NW + C::TW), C::LDS, st);
    return launch_layer<layer_few_kernel<C, false>>(a, C::TM, C::TN, 64 * C::NW, C::LDS, st);
}
template <class C>
static hipError_t launch_ring(const LayerArgs& a, hipStream_t st) {
    if (a.t.P > 0) return launch_layer<layer_ring_kernel<C, true>>(a, C::TM, C::TN, C::THREADS + 64 * C::CW, C::LDS, st);
    return launch_layer<layer_ring_kernel<C, false>>(a, C::TM, C::TN, C::THREADS + 64 * C::CW, C::LDS, st);
}

hipError_t launch_quantised_requests(const QuantisedRequestArgs& a, hipStream_t st) {
    const hipError_t e = a.r.P > 0 ? launch_request_down(a.r, st) : hipSuccess;
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
    int kind = a.r.M <= 16 ? 0 : a.r.M <= 32 ? 1 : a.r.M <= 64 ? 3 : a.r.M <= 256 ? 4 : 6;
    switch (kind) {
        case 0: return launch_few<FewLayer<1, 1, 8, 4, 2>>(g, st);
        case 1: return launch_few<FewLayer<2, 1, 8, 4, 2>>(g, st);
        case 2: return launch_ring<RingLayer<1, 2, 2, 2, 6, 1>>(g, st);        // 32 x 64
        case 3: return launch_ring<RingLayer<2, 2, 2, 2, 7, 2>>(g, st);        // 64 x 64
        case 4: return launch_ring<RingLayer<4, 2, 1, 4, 6, 2>>(g, st);        // 64 x 128
        case 5: return launch_ring<RingLayer<4, 4, 1, 4, 4, 4>>(g, st);        // 64 x 256
        default: return launch_ring<RingLayer<8, 4, 1, 4, 3, 4>>(g, st);       // 128 x 256
    }
}

}  // namespace lf
