// LoRA term of a batch whose rows name their adapters, formed on the accumulators of a wave (lf_gemm_ring.hip: bf16 weights; lf_layer4.hip: 4 bits).
#pragma once
#include "lf_gemm_parts.h"
#include "lf_gemm_ring.h"

namespace lf {

// Distance from matrix instructions written in assembly to the vector ALU's first read of their results.
template <int MI, int NI>
__device__ __forceinline__ void ring_mfma_done(f32x4 (&acc)[MI][NI]) {
    asm volatile("s_nop 15\n\ts_nop 3" ::: "memory");
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) asm volatile("" : "+v"(acc[mi][ni]));
}

// LoRA term of rows with an adapter each, on the accumulators of the wave's MI x NI blocks: a matrix step for every adapter among its rows and
// every 32 columns of its rank (of rank 16 two adapters share a step, each on half of the contraction), with the other rows' S left
// out, on the blocks that have rows of it.  B comes straight from memory in the fragments' layout: an adapter's few rows are read once, by this wave
// alone, DEPTH steps ahead, with no branch around the loads (see ask); S is held in registers.  The steps stand in a list in LDS.  The first of them
// are asked for before the base product where the registers can hold them through it (LATE; the small tiles: 16 rows to a wave), and come in
// meanwhile; elsewhere the whole term comes before the base product, while the copying waves fill the ring.  Bound by the latency of B's
// lines, of which the registers allow four to eight steps under way: 200 rows of 106 adapters, mean rank 37 of 64, 4096 -> 14336: 260 MB, 80 us, of which the
// base product is 39.  us, whole layer, against loads behind branches, whose waits were for all of them, and a list made adapter by adapter: that 103 / 97;
// 64 rows of 48 adapters, r = 16, 4096 -> 6144 19.4 / 17.6; 384 rows of 170, r = 64, 4096 -> 4096 101 / 80; 200 rows, r = 16, 4096 -> 14336 63 / 54;
// 128 rows, r = 32, 4096 -> 4096 27.5 / 25.2.  Steps between the slabs of the base product, two or three ahead, were slower: 103, 21.5, 92, 60, 26.4.
template <class C>
struct RequestList {                                          // of a wave
    static constexpr int ROWS = C::MI * 16;
    int id[ROWS];                                             // adapter of each row, -1: none
    u32x2 unit[2 * ROWS];                                     // adapter; its rank, (8 bits on) the first of the unit's columns, (16 bits on) blocks with rows of it
};
// EVERY > 1: the term is shared out over so many waves with the same rows, this one taking every EVERY-th step from `first` on.
template <class C>
struct RequestTerm {
    static constexpr int MI = C::MI, NI = C::NI, ROWS = MI * 16, EVERY = C::EVERY;
    static_assert(ROWS <= 64, "a lane for every row");
    // what the registers hold beside the accumulators, S and some forty others (LATE: and the fragments of the base product and the term's own
    // accumulators), with two workgroups on a compute unit where the rings allow two (32 x 32 tiles are taken while each has one for itself)
    static constexpr int WAVES = (C::NW + C::CW) * (2 * C::LDS <= 160 * 1024 && C::TN > 32 ? 2 : 1), HOLD = 512 / ((WAVES + 3) / 4) / 8 * 8;
    static constexpr int FRAGS = (C::AHEAD ? 2 * C::SUBS : 2) * (MI + NI) * 4 + MI * NI * 4;
    static constexpr int fit(int beside) { return (HOLD - MI * NI * 4 - MI * 8 - 40 - beside) / (NI * 4 + 2); }
    static constexpr bool LATE = fit(FRAGS) >= 4;
    static constexpr int FIT = fit(LATE ? FRAGS : C::HELD), DEPTH = FIT < 1 ? 1 : FIT > 8 ? 8 : FIT;

    const RingRequestArgs& p;
    const RequestList<C>& list;
    const lora_bf16* s0;
    int n = 0, steps = 0, col0;                               // units, steps of this wave; first column of the wave
    int first;
    int id[MI];
    int row0, rows;                                           // first row of the wave; of the tile
    uint32_t boff[NI];                                        // (32-bit offsets within an adapter: N <= 2^22, r <= 64)
    bf16x8 s[2][MI];                                          // the rows' S: columns 8 q .. of the first 32 and of the others; r = 16: 8 (q & 1) ..
    u32x4 b[DEPTH][NI];
    u32x2 e[DEPTH];                                           // the lane's unit

    __device__ __forceinline__ RequestTerm(const RingRequestArgs& args, const RowTile& rt, int c0, int wm, int wn, RequestList<C>& out,
                                           int from = 0)
        : p(args), list(out), s0(args.ltok + (int64_t)rt.row_start * args.lr), col0(c0 + wn * NI * 16), first(from), row0(wm * ROWS), rows(rt.rows) {
        const int l = threadIdx.x & 63, q = l >> 4, width = p.lr == 16 ? 16 : 32;
        const int row = wm * ROWS + l;
        int of = p.ids[rt.row_start + min(row, rt.rows - 1)];
        if (l >= ROWS || row >= rt.rows || of >= p.P || of < 0) of = -1;
        const int rank = of < 0 ? 0 : p.ranks ? max(min(p.ranks[of], p.lr), 0) : p.lr;
        // the rows of each row's adapter, from the bits of their numbers; the first of them enters it
        uint64_t its = __ballot(rank > 0);
        if (!its) return;
        for (int bit = 0; (p.P - 1) >> bit; ++bit) {
            const bool set = of >> bit & 1;
            const uint64_t all = __ballot(set);
            its &= set ? all : ~all;
        }
        const uint64_t below = (1ull << l) - 1;
        const bool enters = rank > 0 && !(its & below), more = enters && rank > 32;
        const uint64_t in = __ballot(enters), in2 = __ballot(more);
        const int at = __popcll(in & below) + __popcll(in2 & below);
        n = __popcll(in) + __popcll(in2);
        if (l < ROWS) out.id[l] = of;
        if (enters) {
            uint32_t blocks = 0;
#pragma unroll
            for (int mi = 0; mi < MI; ++mi) blocks |= (its >> (16 * mi) & 0xFFFFu) ? 1u << mi : 0u;
            out.unit[at] = u32x2{(uint32_t)of, (uint32_t)rank | blocks << 16};
            if (more) out.unit[at + 1] = u32x2{(uint32_t)of, (uint32_t)rank | 32u << 8 | blocks << 16};
        }
        steps = width == 16 ? (n + 1) / 2 : n;
        if constexpr (EVERY > 1) steps = max(steps - first + EVERY - 1, 0) / EVERY;
        asm volatile("" ::: "memory");                        // (LDS operations of a wave complete in order)
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            id[mi] = list.id[mi * 16 + (l & 15)];
            const uint32_t soff = s_row(mi, l);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = width == 16 ? 8 * (q & 1) : 32 * h + 8 * q;
                const u32x4 v = *(const u32x4*)(s0 + soff + (k < p.lr ? k : 0));
                s[h][mi] = __builtin_bit_cast(bf16x8, k < p.lr ? v : u32x4{0u, 0u, 0u, 0u});
            }
        }
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) boff[ni] = (uint32_t)min(col0 + ni * 16 + (l & 15), p.NC - 1) * p.lr + own_column();
#pragma unroll
        for (int t = 0; t < DEPTH; ++t) ask(t, unit_of(t));
    }

    __device__ __forceinline__ uint32_t s_row(int mi, int l) const { return (uint32_t)min(row0 + mi * 16 + (l & 15), rows - 1) * p.lr; }

    // A lane's unit in a step (past the last one: that one, with nothing of it), and how many entries of its eight the adapter has there.
    __device__ __forceinline__ u32x2 unit_of(int step) const {
        if constexpr (EVERY > 1) step = first + step * EVERY;
        const int u = p.lr == 16 ? 2 * step + ((threadIdx.x & 63) >> 5) : step;
        u32x2 v = list.unit[min(u, n - 1)];
        if (u >= n) v.y = 0u;
        return v;
    }
    __device__ __forceinline__ int own_column() const { const int q = (threadIdx.x & 63) >> 4; return p.lr == 16 ? 8 * (q & 1) : 8 * q; }
    static __device__ __forceinline__ int column_of(uint32_t y) { return (int)(y >> 8 & 0xFFu); }
    __device__ __forceinline__ int left_of(uint32_t y) const { return (int)(y & 0xFFu) - column_of(y) - own_column(); }

    // B of a step, into place t.  Without a branch, since behind one the waits for what was asked for before are waits for everything.
    __device__ __forceinline__ void ask(int t, u32x2 unit) {
        const char* bg = (const char*)p.lout + ((uint64_t)unit.x * (uint32_t)(2 * p.NC * p.lr) + 2 * column_of(unit.y));
        e[t] = unit;
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) b[t][ni] = *(const u32x4*)(bg + 2 * (uint64_t)boff[ni]);
    }

    // The matrix steps of place t, for the blocks that have rows of its adapters.  CLEAR: with 0 for what is not finite in B.
    template <bool CLEAR>
    __device__ __forceinline__ void step_at(f32x4 (&acc)[MI][NI], int t) {
        const int left = left_of(e[t].y);
        if (__any(left < 8))
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t m = 2 * i + 1 < left ? 0xFFFFFFFFu : 2 * i < left ? 0xFFFFu : 0u;
#pragma unroll
                for (int ni = 0; ni < NI; ++ni) b[t][ni][i] &= m;
            }
        if constexpr (CLEAR)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = b[t][ni][i];
                    b[t][ni][i] = ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
                }
        const uint32_t y = (uint32_t)__builtin_amdgcn_readlane((int)e[t].y, 0), blocks = (y | (uint32_t)__builtin_amdgcn_readlane((int)e[t].y, 32)) >> 16;
        const bool second = y >> 13 & 1;                      // columns 32 and further
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
            if (!(blocks >> mi & 1)) continue;
            const bf16x8 v = second ? s[1][mi] : s[0][mi];
            const bf16x8 own = id[mi] == (int)e[t].x ? v : bf16x8{};
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = LF_MFMA(__builtin_bit_cast(bf16x8, b[t][ni]), own, acc[mi][ni]);
        }
    }

    // The term; acc comes in as zeros.
    __device__ __forceinline__ void form(f32x4 (&acc)[MI][NI]) {
        if (!steps) return;
        u32x2 next = unit_of(DEPTH);
        int step = 0;
        for (; step + DEPTH < steps; step += DEPTH) {
#pragma unroll
            for (int t = 0; t < DEPTH; ++t) {
                const u32x2 unit = next;
                next = unit_of(step + t + DEPTH + 1);
                step_at<false>(acc, t);
                ask(t, unit);
            }
        }
#pragma unroll
        for (int t = 0; t < DEPTH; ++t)
            if (step + t < steps) step_at<false>(acc, t);
        ring_mfma_done<MI, NI>(acc);                          // (across the blocks that are passed over the compiler keeps no distance)
        // infinity or NaN in an adapter's B has met the zeros of the block's other rows: those are done again
        float bad = 0.f;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                for (int i = 0; i < 4; ++i) bad = __builtin_fmaf(acc[mi][ni][i], 0.f, bad);
        if (__any(bad != 0.f)) again(acc);
    }

    // ... with what is not finite in B left out, then added to the rows that have the adapter.
    __device__ __forceinline__ void again(f32x4 (&acc)[MI][NI]) {
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int step = 0; step < steps; ++step) {
            ask(0, unit_of(step));
            step_at<true>(acc, 0);
        }
        ring_mfma_done<MI, NI>(acc);
#pragma unroll 1
        for (int u = 0; u < n; ++u) {
            if (EVERY > 1 && (p.lr == 16 ? u / 2 : u) % EVERY != first) continue;
            const u32x2 unit = list.unit[u];
            const int g = (int)unit.x, k0 = column_of(unit.y);
#pragma unroll 1
            for (int k = k0; k < min((int)(unit.y & 0xFFu), k0 + (p.lr == 16 ? 16 : 32)); ++k) {
                int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
                asm volatile("" : "+v"(l));                   // (so that nothing derived from it is kept through the loops)
                float sk[MI];
#pragma unroll
                for (int mi = 0; mi < MI; ++mi) sk[mi] = __builtin_bit_cast(float, (uint32_t)s0[s_row(mi, l) + k] << 16);
#pragma unroll
                for (int ni = 0; ni < NI; ++ni)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        __builtin_amdgcn_sched_barrier(0);
                        const int64_t col = min(col0 + ni * 16 + 4 * (l >> 4) + i, p.NC - 1);
                        const float x = __builtin_bit_cast(float, (uint32_t)p.lout[((int64_t)g * p.NC + col) * p.lr + k] << 16);
                        const bool odd = (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) == 0x7F800000u;
#pragma unroll
                        for (int mi = 0; mi < MI; ++mi) acc[mi][ni][i] += odd && id[mi] == g ? sk[mi] * x : 0.f;
                    }
            }
        }
    }
};
}  // namespace lf
