// The LoRA linear layer for many requests over 4-bit weights:
//     S[i] = s_g X[i] A_g^T             lf_requests.hip; of a few short rows here (own_term)
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
    const lora_bf16* A; const float* s; lora_bf16* S;      // where the layer forms S by itself
};

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

// Copies of rows of 16-byte chunks, N of 1 KB, to `to`; off: biased (kCopyBias, pass_imm).
template <int N, int I = 0>
__device__ __forceinline__ void copy_rows(const char* biased, const uint32_t (&off)[N], uint32_t to) {
    if constexpr (I < N) {
        copy16_to_lds<pass_imm(N, I), I == 0>(biased, off[I], to + N / 2 * 1024);
        copy_rows<N, I + 1>(biased, off, to);
    }
}
// Position of 16-byte chunk ch of a row: of X (256 bytes), where the 16 rows of a fragment need 16 positions; of codes (64 bytes), where four rows share 256 bytes.
__device__ __forceinline__ int x_chunk(int row, int ch) { return ch ^ (row & 15); }
__device__ __forceinline__ int code_chunk(int row, int ch) { return ch ^ (row >> 2 & 3); }

// What one wave brings of a block into LDS, and how: XC x 4 rows of X to `x`; CC x 16 rows of codes from row c0 + first on to `part`, behind them their exponents (four bytes a
// row, for 64 lanes) and, SPLIT, the four bytes behind those: where rows are not whole blocks every other row's block starts in the middle of four bytes.
template <int XC, int CC, bool SPLIT>
struct BlockCopies {
    static constexpr int N = XC + CC + (SPLIT ? 2 : 1), RW = 16 * CC, PART = RW * (kBlock / 2) + 512;
    static constexpr int AT = (CC - CC / 2) * 1024;            // M0 stands in the middle of the codes: the exponents' immediates count from there
    const LayerArgs& p;
    int x_row, x_rows, first, c0, whole;
    uint32_t xo[XC], co[CC], eo, left;
    const char* x;
    const char* codes;
    const char* exps;

    // x_first: of the wave's rows of X in the tile; code_first: of its rows of codes
    __device__ __forceinline__ BlockCopies(const LayerArgs& args, const RowTile& rt, int tile_c0, int x_first, int code_first)
        : p(args), x_row(x_first), x_rows(rt.rows), first(code_first), c0(tile_c0), whole(args.t.KC / kBlock) {
        const int l = threadIdx.x & 63, K = p.t.KC;
        form(kBlock / 2);
        eo = (uint32_t)min(first + l % RW, p.t.NC - 1 - c0) * (uint32_t)(K / 32) + kCopyBias - AT;
        x = (const char*)(p.t.tok + (int64_t)rt.row_start * K) - kCopyBias;
        codes = (const char*)p.codes + (int64_t)c0 * (K / 2) - kCopyBias;
        exps = (const char*)p.exps + (int64_t)c0 * (K / 32) - kCopyBias;
        left = (uint32_t)min((int64_t)(p.t.NC - c0) * (K / 32), (int64_t)1 << 30);      // to the array's end, from the tile's first row
    }
    __device__ __forceinline__ void form(int bytes) {          // valid bytes of a row of codes
        const int l = threadIdx.x & 63, K = p.t.KC;
#pragma unroll
        for (int i = 0; i < XC; ++i) {
            const int row = x_row + 4 * i + l / 16, ch = min(x_chunk(row, l % 16), bytes / 4 - 1);
            xo[i] = ((uint32_t)min(row, x_rows - 1) * (uint32_t)K + 8 * ch) * 2 + kCopyBias - pass_imm(XC, i);
        }
#pragma unroll
        for (int i = 0; i < CC; ++i) {
            const int row = first + 16 * i + l / 4, ch = min(code_chunk(row, l % 4), bytes / 16 - 1);
            co[i] = (uint32_t)min(row, p.t.NC - 1 - c0) * (uint32_t)(K / 2) + 16 * ch + kCopyBias - pass_imm(CC, i);
        }
    }
    __device__ __forceinline__ void block(int b, uint32_t x_to, uint32_t part_to) {
        if (b >= whole) form(kBlock / 4);
        copy_rows<XC>(x + (int64_t)b * (2 * kBlock), xo, __builtin_amdgcn_readfirstlane(x_to));
        copy_rows<CC>(codes + (int64_t)b * (kBlock / 2), co, __builtin_amdgcn_readfirstlane(part_to));
        const char* e = exps + (int64_t)b * (kBlock / 32);
        if constexpr (SPLIT) {
            // the offsets are even, from an array whose start is a multiple of 16, as is the tile's first row
            const uint32_t at = eo - (kCopyBias - AT) + b * (kBlock / 32), down = at & 2u, behind = min(at - down + 4, left - 4);
            copy4_to_lds<AT>(e, eo - down);
            copy4_to_lds<AT + 256>(exps, behind + kCopyBias - AT - 256);
        } else {
            copy4_to_lds<AT>(e, eo);
        }
    }
};
// Byte of a lane's exponent behind the codes of its part, row r of it (c = r & 15); half: of the half block at the end.
__device__ __forceinline__ int exp_byte(bool split, int r, int c, int q) { return 4 * r + (split && (c & 1) ? (q < 2 ? 2 + q : 256 - 2 + q) : q); }
__device__ __forceinline__ int half_exp_byte(int r, int c, int q) { return 4 * r + 2 * (c & 1) + (q >> 1); }

// ---- few rows ---------------------------------------------------------------------------------------
// Bound by what a compute unit brings in, of which a launch of a few us sees mostly the latency: X comes again with every tile of columns, beside 1 KB of codes of a 16 x 16 tile's
// block 4 KB of it (1 KB where there are four rows at most).  Without adapters, in a captured graph, 14336 -> 4096: one row 8.6 us, four 8.5, five 10.3, 16 rows 11.7, 64 rows (16 x 64
// tiles) 19.9, that is 49 and 47 KB a us and compute unit for the last two; 4096 -> 4096 4.2, 4.4, 4.7, 5.3, 7.8.
// A workgroup has up to 16 rows (of which it brings 4 XC) and NI x 16 columns, its NW waves every NW-th block of the contraction, which each brings into a ring of
// its own of D blocks, with no barrier; the adapters' term is formed by TW waves of its own beside them, which share its steps.  Sums of the waves are added in LDS
// in a fixed order.  Measured (us, in a captured graph, the first product's launch included where there are adapters): one row 4096 -> 14336, r = 16, 12.2 (31 MB of weights; without adapters 8.4; codes
// from memory straight into the lanes that use them 22); 16 rows 4096 -> 6144, no adapters 6.0, 12 of r = 16 10.1; 16 rows 14336 -> 4096 11.7 and 17.2.  Three blocks
// to a ring of the 16 x 32 tiles instead of two, which is all that LDS holds: the same.
template <int XC_, int NI_, int NW_, int TW_, int D_>
struct FewLayer {
    static constexpr bool FEW = true;
    static constexpr int XC = XC_, NI = NI_, NW = NW_, TW = TW_, D = D_, TN = 16 * NI;
    struct Term {                      // of one wave
        static constexpr int MI = 1, NI = NI_, NW = NW_, CW = TW_, LDS = 160 * 1024, TN = 16 * NI_, SUBS = 0, EVERY = TW_, HELD = 0;
        static constexpr bool AHEAD = false;
    };
    static constexpr int SLOT = XC * 1024 + BlockCopies<XC, NI, true>::PART;
    static constexpr int TM = 16, RING_BLOCKS = NW * D;
    static constexpr int RING = NW * D * SLOT, SUMS = (NW + TW) * NI * 1024, BODY = RING > SUMS ? RING : SUMS;
    static constexpr int LDS = BODY + TW * (int)sizeof(RequestList<Term>);
    static_assert((XC + NI + 2) * (D - 1) < 64 && LDS <= 160 * 1024, "the wait counter; a compute unit's LDS");
};

template <class C, bool SPLIT>
__device__ __forceinline__ void few_products(const LayerArgs& p, const RowTile& rt, int c0, int w, char* ring, f32x4 (&acc)[1][C::NI]) {
    constexpr int NI = C::NI, D = C::D;
    using Copies = BlockCopies<C::XC, NI, SPLIT>;
    const int l = threadIdx.x & 63, c = l & 15, q = l >> 4, blocks = (p.t.KC + kBlock - 1) / kBlock;
    Copies copies(p, rt, c0, 0, 0);
    const uint32_t lds = lds_addr_of(ring);
    const int xr = min(c, 4 * C::XC - 1);                      // (rows past those there are: results that are not stored)
    auto ask = [&](int b, int slot) {
        if (b < blocks) copies.block(b, lds + slot * C::SLOT, lds + slot * C::SLOT + C::XC * 1024);
    };
#pragma unroll
    for (int d = 0; d < D; ++d) ask(w + C::NW * d, d);
    int slot = 0;
    for (int b = w; b < blocks; b += C::NW) {
        if (b + C::NW * (D - 1) < blocks) wait_slab_loads_but<Copies::N*(D - 1)>();
        else wait_slab_loads();
        const char* st = ring + slot * C::SLOT;
        const char* part = st + C::XC * 1024;
        if (!SPLIT || b < copies.whole) {
            bf16x8 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __builtin_bit_cast(bf16x8, *(const u32x4*)(st + xr * 256 + (x_chunk(xr, 4 * q + j) << 4)));
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const u32x4 cd = *(const u32x4*)(part + (16 * ni + c) * 64 + (code_chunk(c, q) << 4));
                const float sc = exp2_of_biased(*(const uint8_t*)(part + Copies::RW * 64 + exp_byte(SPLIT, 16 * ni + c, c, q)));
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[0][ni] = LF_MFMA(from_fp4(cd[j], sc), x[j], acc[0][ni]);
            }
        } else {                                               // half a block, in two steps: 16 entries of each row to a lane
            bf16x8 x[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) x[j] = __builtin_bit_cast(bf16x8, *(const u32x4*)(st + xr * 256 + (x_chunk(xr, 2 * q + j) << 4)));
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const u32x4 cd = *(const u32x4*)(part + (16 * ni + c) * 64 + (code_chunk(c, q >> 1) << 4));
                const float sc = exp2_of_biased(*(const uint8_t*)(part + Copies::RW * 64 + half_exp_byte(16 * ni + c, c, q)));
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[0][ni] = LF_MFMA(from_fp4(q & 1 ? cd[2 + j] : cd[j], sc), x[j], acc[0][ni]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (the block is read: its place is free)
        ask(b + C::NW * D, slot);
        slot = slot + 1 == D ? 0 : slot + 1;
    }
}

// S and the term of a few rows in one go, in wave t of TW: each wave has its part of the adapter's columns, whose S it forms (in fp32, rounded to bf16 as where it is stored) and
// multiplies with its part of B.  Every workgroup reads the rows' A for itself, row after row and four columns at a time, which has to be less than a launch of its own (launch_quantised_requests).
template <class C>
__device__ __forceinline__ void own_term(const LayerArgs& p, const RowTile& rt, int c0, int t, f32x4 (&acc)[1][C::NI]) {
    const int l = threadIdx.x & 63, c = l & 15, q = l >> 4, K = p.t.KC, r = p.t.lr, own = r / C::TW;
    for (int i = 0; i < rt.rows; ++i) {
        const int64_t row = rt.row_start + i;
        const int g = __builtin_amdgcn_readfirstlane(p.t.ids[row]);
        const bool has = g >= 0 && g < p.t.P;
        const int rank = has ? p.t.ranks ? max(min(__builtin_amdgcn_readfirstlane(p.t.ranks[g]), r), 0) : r : 0;
        const float s = has ? p.s[g] : 0.f;
        for (int j = t * own; j < (t + 1) * own; j += 4) {
            u32x2 held = u32x2{0u, 0u};
            if (j < rank) {
                u32x2 b[C::NI][4];
#pragma unroll
                for (int ni = 0; ni < C::NI; ++ni)
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        if (c == i) b[ni][n] = *(const u32x2*)(p.t.lout + ((int64_t)g * p.t.NC + c0 + 16 * ni + 4 * q + n) * r + j);
                const lora_bf16* x = p.t.tok + row * K;
                const lora_bf16* a = p.A + ((int64_t)g * r + j) * K;
                float d[4] = {0.f, 0.f, 0.f, 0.f}, v[4];
#pragma unroll 2
                for (int k = 8 * l; k < K; k += 512) {
                    float xf[8];
                    unpack8(*(const u32x4*)(x + k), xf);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        float af[8];
                        unpack8(*(const u32x4*)(a + (int64_t)u * K + k), af);
#pragma unroll
                        for (int e = 0; e < 8; ++e) d[u] += xf[e] * af[e];
                    }
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
#pragma unroll
                    for (int o = 32; o > 0; o >>= 1) d[u] += __shfl_xor(d[u], o);
                    v[u] = j + u < rank ? s * d[u] : 0.f;
                }
                held = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                if (c == i)
#pragma unroll
                    for (int ni = 0; ni < C::NI; ++ni)
#pragma unroll
                        for (int n = 0; n < 4; ++n)
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const uint32_t sh = u & 1 ? 0u : 16u;
                                const float su = __builtin_bit_cast(float, held[u / 2] << sh & 0xFFFF0000u), bu = __builtin_bit_cast(float, b[ni][n][u / 2] << sh & 0xFFFF0000u);
                                if (j + u < rank) acc[0][ni][n] += su * bu;
                            }
            }
            if (c0 == 0 && l == 0) *(u32x2*)(p.S + row * r + j) = held;
        }
    }
}

enum class Few { plain, term, own };           // no adapters; their S from memory; formed here
template <class C, Few FORM>
__global__ void __launch_bounds__(64 * (C::NW + (FORM != Few::plain ? C::TW : 0))) layer_few_kernel(LayerArgs p) {
    constexpr bool TERM = FORM != Few::plain;
    constexpr int NI = C::NI, NW = C::NW, WAVES = NW + (TERM ? C::TW : 0);
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;
    const int c0 = (int)blockIdx.x % p.t.tiles_n * C::TN;
    RowTile rt{};
    rt.row_start = p.t.row_lo + (int)blockIdx.x / p.t.tiles_n * 16;
    rt.rows = min(16, p.t.row_hi - rt.row_start);
    f32x4 acc[1][NI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) acc[0][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (FORM == Few::own && w >= NW) {
        own_term<C>(p, rt, c0, w - NW, acc);
    } else if (TERM && w >= NW) {
        using T = typename C::Term;
        RequestTerm<T> term(p.t, rt, c0, 0, 0, ((RequestList<T>*)(smem + C::BODY))[w - NW], w - NW);
        term.form(acc);
    } else if (p.t.KC % kBlock) {
        few_products<C, true>(p, rt, c0, w, smem + w * C::D * C::SLOT, acc);
    } else {
        few_products<C, false>(p, rt, c0, w, smem + w * C::D * C::SLOT, acc);
    }
    __syncthreads();
    f32x4* sums = (f32x4*)smem;                                // [wave][ni][lane]
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) sums[(w * NI + ni) * 64 + l] = acc[0][ni];
    __syncthreads();
    if (w >= NI) return;
    f32x4 y = sums[w * 64 + l];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) y += sums[(i * NI + w) * 64 + l];
    if (c < rt.rows) *(u32x2*)(p.t.res + (int64_t)(rt.row_start + c) * p.t.NC + c0 + 16 * w + 4 * q) = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

// ---- more rows --------------------------------------------------------------------------------------
// X, the codes and the exponents go through a ring of NS blocks in LDS, filled by CW waves that do nothing else.  A wave's 16 MI x 16 NI tile is one stream of
// instructions over the blocks: a matrix instruction to a slot, and between them the reads of the fragments of X, three ahead of their use, and the widening of the next
// step's codes.  (Codes straight from memory into the registers of the lanes that use them, 16 bytes of a row to each: neighbouring lanes have other rows, so that a
// load takes 64 cycles of the address unit instead of 16, and one of exponents, a byte to a lane, as many; 2048 rows, 4096 -> 4096: 71 us, 1.9 us a block; this 50, 1363 TFLOP/s.)  The term comes before the first block, while the ring is
// filled: 96 rows of 64 adapters, r = 64, 4096 -> 14336: 42 us with it, 18 without.  Formed meanwhile by waves of its own, four or eight, which meet the others at the ring's barriers, with
// B in registers or through LDS, a row's 64 bytes to four lanes: 40, and 5 - 8 % more than now for adapters of r = 16, K = 1024; it is B's lines that take the
// time, 95 MB in pieces of 64 bytes.
template <int MI_, int NI_, int WM_, int WN_, int NS_, int CW_>
struct RingLayer {
    static constexpr bool FEW = false;
    static constexpr int MI = MI_, NI = NI_, WM = WM_, WN = WN_, NS = NS_, CW = CW_, NW = WM * WN, THREADS = 64 * NW;
    static constexpr int TM = 16 * MI * WM, TN = 16 * NI * WN;
    static constexpr int XB = TM * 2 * kBlock, XC = XB / 1024 / CW, RW = TN / CW, CC = RW / 16;     // a block's X, then the parts of the copying waves
    static constexpr int PART = BlockCopies<XC, CC, true>::PART, STAGE = XB + CW * PART;
    static constexpr int OUT = TM * TN * 2;
    static constexpr int HALVES = (MI + 3) / 4;                                     // the term is formed for 64 rows of a wave at a time
    struct Term {
        static constexpr int MI = MI_ > 4 ? MI_ / 2 : MI_, NI = NI_, NW = WM_ * WN_, CW = CW_, LDS = NS_ * STAGE, TN = 16 * NI_ * WN_, SUBS = 2, EVERY = 1;
        static constexpr int HELD = (MI_ - MI) * NI * 4;                            // the other rows' accumulators
        static constexpr bool AHEAD = false;
    };
    static constexpr int RING_BLOCKS = NS;
    static constexpr int RING = NS * STAGE > OUT ? NS * STAGE : OUT;
    static constexpr int LDS = RING + NW * (int)sizeof(RequestList<Term>);
    static_assert(XB % (1024 * CW) == 0 && XC <= 8 && RW % 16 == 0 && RW <= 64, "copies of a block: whole, in reach of the immediates");
    static_assert((XC + CC + 2) * (NS - 2) < 64, "... and of the wait counter");
    static_assert(NS >= 3 && LDS <= 160 * 1024, "a compute unit's LDS");
};
// The copying waves.  Block b + NS - 1 goes where block b - 1 was, which every wave has left when it comes to the barrier in block b; behind that barrier block
// b + 1 has landed.
template <class C, bool SPLIT>
__device__ __forceinline__ void copying_wave(const LayerArgs& p, const RowTile& rt, int c0, int w, uint32_t lds) {
    constexpr int NS = C::NS;
    using Copies = BlockCopies<C::XC, C::CC, SPLIT>;
    Copies copies(p, rt, c0, w * C::XC * 4, w * C::RW);
    const int whole = copies.whole, blocks = (p.t.KC + kBlock - 1) / kBlock;
    auto block = [&](int b, int stage) {
        if (b < blocks) copies.block(b, lds + stage * C::STAGE + w * C::XC * 1024, lds + stage * C::STAGE + C::XB + w * C::PART);
    };
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) block(s, s);
    if (blocks >= NS - 1) wait_slab_loads_but<Copies::N*(NS - 2)>();
    else wait_slab_loads();
    asm volatile("s_barrier" ::: "memory");
    int stage = NS - 1;
    for (int b = 0; b < whole; ++b) {
        if (b + NS - 1 <= blocks) wait_slab_loads_but<Copies::N*(NS - 3)>();
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
        const bool split = blocks > whole;
        auto read_codes = [&](int stage, int ni) {
            coming[ni] = *(const u32x4*)(part_of(stage, ni) + row_of(ni) * 64 + (code_chunk(c, q) << 4));
        };
        auto read_exp = [&](int stage, int ni) {
            e[ni] = *(const uint8_t*)(part_of(stage, ni) + C::RW * 64 + exp_byte(split, row_of(ni), c, q));
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
                const float sc = exp2_of_biased(*(const uint8_t*)(part + C::RW * 64 + half_exp_byte(row_of(ni), c, q)));
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
static hipError_t launch_kind(const LayerArgs& a, bool own, hipStream_t st) {
    if constexpr (C::FEW) {
        constexpr int THREADS = 64 * (C::NW + C::TW);
        if constexpr (C::XC == 1)
            if (own) return launch_layer<layer_few_kernel<C, Few::own>>(a, 16, C::TN, THREADS, C::LDS, st);
        if (a.t.P > 0) return launch_layer<layer_few_kernel<C, Few::term>>(a, 16, C::TN, THREADS, C::LDS, st);
        return launch_layer<layer_few_kernel<C, Few::plain>>(a, 16, C::TN, 64 * C::NW, C::LDS, st);
    } else {
        if (a.t.P > 0) return launch_layer<layer_ring_kernel<C, true>>(a, C::TM, C::TN, C::THREADS + 64 * C::CW, C::LDS, st);
        return launch_layer<layer_ring_kernel<C, false>>(a, C::TM, C::TN, C::THREADS + 64 * C::CW, C::LDS, st);
    }
}

// Rows and columns of a workgroup, and what a block of the contraction takes it, us, while there is one on a compute unit; 2.5 a round beside them (fitted to 1 - 2048
// rows, K of 1024 - 14336, N of 1024 - 14336).  The first three are layer_few_kernel.
struct LayerKind { int rows, columns; float block; };
constexpr LayerKind kLayerKinds[] = {{16, 16, 0.085f}, {16, 32, 0.098f}, {16, 64, 0.152f}, {32, 64, 0.25f}, {64, 64, 0.30f}, {64, 128, 0.43f}, {64, 256, 0.62f},
                                     {128, 256, 1.08f}};
static int choose_kind(int M, int K, int N) {
    int best = 0;
    float least = 0.f;
    for (int i = 0; i < (int)(sizeof(kLayerKinds) / sizeof(kLayerKinds[0])); ++i) {
        const LayerKind& k = kLayerKinds[i];
        const int64_t tiles = (int64_t)((M + k.rows - 1) / k.rows) * ((N + k.columns - 1) / k.columns);
        const float us = (float)((tiles + kComputeUnits - 1) / kComputeUnits) * (2.5f + k.block * (float)K / kBlock);
        if (i == 0 || us < least) {
            least = us;
            best = i;
        }
    }
    return best;
}

// f(kind): of the layer over these rows.
template <class F>
static auto with_kind(int M, int K, int N, F&& f) {
    switch (choose_kind(M, K, N)) {
        case 0: return M <= 4 ? f(FewLayer<1, 1, 8, 4, 4>{}) : f(FewLayer<4, 1, 8, 4, 3>{});
        case 1: return f(FewLayer<4, 2, 8, 4, 2>{});
        case 2: return f(FewLayer<4, 4, 8, 4, 2>{});
        case 3: return f(RingLayer<1, 2, 2, 2, 6, 1>{});
        case 4: return f(RingLayer<2, 2, 2, 2, 7, 2>{});
        case 5: return f(RingLayer<4, 2, 1, 4, 6, 2>{});
        case 6: return f(RingLayer<4, 4, 1, 4, 4, 4>{});
        default: return f(RingLayer<8, 4, 1, 4, 3, 4>{});
    }
}

// S formed by every workgroup for itself (own_term), where its rows' columns are few and short enough.  us in a captured graph (with the call from Python), two
// launches / one: one row of r = 16, 1024 -> 1024 5.7 / 3.9 (9.6 / 7.3), 4096 -> 4096 7.5 / 6.8 (9.7 / 7.3), 8192 -> 2048 9.8 / 10.1; of 32, 1024 -> 1024 5.8 / 4.7,
// 2048 -> 4096 6.5 / 7.1; of 64, 256 -> 256 5.8 / 5.6, 1024 -> 1024 6.1 / 6.3; two of 16, 1024 -> 1024 6.0 / 5.0, 2048 -> 4096 6.5 / 7.3.  (With wider tiles, N = 14336, it was
// never faster: 12.2 / 18.2 for one row of 4096.)
static bool forms_own_term(int M, int K, int N, int r, int P) {
    const int64_t columns = (int64_t)M * r;
    return P > 0 && M <= 4 && choose_kind(M, K, N) == 0 && columns * columns * K <= 1 << 20;
}

QuantisedTiles quantised_tiles(int M, int K, int N, int r, int P) {
    return with_kind(M, K, N, [&](auto c) { return QuantisedTiles{c.TM, c.TN, c.RING_BLOCKS, forms_own_term(M, K, N, r, P)}; });
}

hipError_t launch_quantised_requests(const QuantisedRequestArgs& a, hipStream_t st) {
    const bool own = forms_own_term(a.r.M, a.r.K, a.r.N, a.r.r, a.r.P);
    const hipError_t e = a.r.P > 0 && !own ? launch_request_down(a.r, st) : hipSuccess;
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
    if (own) {
        g.A = a.r.A;
        g.s = a.r.s;
        g.S = a.r.S;
    }
    return with_kind(a.r.M, a.r.K, a.r.N, [&](auto c) { return launch_kind<decltype(c)>(g, own, st); });
}

}  // namespace lf
