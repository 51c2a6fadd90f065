// Attention of the new tokens of each sequence over a paged cache that holds them already:
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - m),  over the keys j <= pos, with a window j > pos - window,
// one pass over the keys with the running maximum m and sum of the softmax in fp32.  Grouped heads: the rows of a tile are (token, query
// head of one key/value head), so that what is read of the cache serves all of them.
//
// Scores are formed transposed, S^T = K Q^T, and so is the result, O^T = V^T P^T: a lane then holds of one query (its column, l & 15)
// the scores of four keys of every block of 16, which is how the second product takes its operand, if the 32 keys of a matrix step are
// numbered as the lanes hold them (keys 4q .. 4q+3 and 16+4q .. 16+4q+3 for the lanes with l >> 4 = q): P goes from one product to the
// other in registers, a maximum is taken over the registers and two lane exchanges, and V's transposed fragments come from LDS with
// transposing reads.
//
// Two kernels.  Few rows (attn_few_kernel: decoding and short chunks, 16 or 32 rows): bound by the reading of the cache; each of a
// workgroup's four waves goes through keys of its own, K straight into fragments, V through LDS of the wave's own, no barrier;
// sums are joined at the end.  Many rows (attn_many_kernel, 128 rows): bound by the matrix and vector work; the four waves share tiles of 64
// keys in LDS, 32 rows to a wave.  Long key ranges of few tiles are cut into parts for more workgroups, whose results
// attn_join_kernel adds.
//
// The fp8 form of the cache is widened to bf16 (exact: e4m3 times a power of two) on the way to LDS or into the fragments.
#include <algorithm>
#include <type_traits>

#include "lf_gemm_parts.h"
#include "lf_serve.h"

namespace lf {

constexpr float kNone = -__FLT_MAX__;             // reference of a row that has seen nothing: finite, so that every p against it is 0 and no case of its own
constexpr float kFar = 0x1p20f;                  // the largest reference that p is formed against in one step (move_base)

// What a workgroup works on.
struct AttnTile {
    int b, g, tile, split;             // sequence, key/value head, row tile, part of the keys
    int first, n, kv;                  // first row of the sequence's new tokens, their number, length with them
    int row0, rows;                    // first (token, head) row of the tile and how many it has
    int key_lo, key_hi;                // keys that any of its rows sees; key_lo a multiple of 16
    int k0, k1;                        // ... and of them this part's
    int parts;                         // parts that have keys (at least 1)
};

template <int BM>
__device__ __forceinline__ bool attn_rows(const AttnArgs& p, AttnTile& t) {
    t.first = min(max(p.offsets[t.b], 0), p.T);
    t.n = min(p.offsets[t.b + 1], p.T) - t.first;
    t.kv = max(min(p.kv_lens[t.b], p.max_pages << p.c.page_shift), 0);
    t.row0 = t.tile * BM;
    t.rows = min(BM, max(t.n, 0) * p.group - t.row0);
    if (t.rows <= 0) return false;
    const int t_lo = t.row0 / p.group, t_hi = (t.row0 + t.rows - 1) / p.group;
    t.key_hi = max(t.kv - t.n + t_hi + 1, 0);
    t.key_lo = p.window ? max(t.kv - t.n + t_lo - p.window + 1, 0) & ~15 : 0;
    t.parts = min(max((t.key_hi - t.key_lo + p.split_keys - 1) / p.split_keys, 1), p.splits);
    return true;
}

template <int BM>
__device__ __forceinline__ bool attn_tile(const AttnArgs& p, AttnTile& t) {
    // Key/value heads of a sequence fastest: with eight heads the tiles that share keys are on one XCD.  Then tiles, the last first, since they see the
    // most keys; parts slowest: the last ones, which hold what is left of a range, run last.  Within an XCD workgroups go to its four
    // shader engines in turn, full or not: with sequences before tiles, two of them (5003 and 16000 keys, 1021 new tokens) left half
    // the engines without work for half of the time (515 us instead of 363).  Every part starts at another sequence, so that the parts of a long
    // one are not all on the same compute units (this launch and the join, us: 300 -> 275; four sequences of 33000 - 131072, few rows: 260 -> 254).
    int id = blockIdx.x;
    t.g = id % p.c.heads;
    id /= p.c.heads;
    t.tile = p.tiles - 1 - id % p.tiles;
    id /= p.tiles;
    t.b = id % p.B;
    t.split = id / p.B;
    t.b = (t.b + t.split * (p.B / 4 + 1)) % p.B;
    if (!attn_rows<BM>(p, t) || t.split >= t.parts) return false;
    t.k0 = t.key_lo + t.split * p.split_keys;
    t.k1 = t.split + 1 == p.splits ? t.key_hi : min(t.key_hi, t.k0 + p.split_keys);     // (the last takes what there is: lengths past max_kv)
    return true;
}

// Page of a 16-key block that starts at `key` (below the length, the same for the whole wave), as the table has it: a scalar load, asked for a step
// before it is needed.  A vector load, with the wait for it before the step's copies could be issued, took a third of the time.
__device__ __forceinline__ int page_of(const AttnArgs& p, const AttnTile& t, int key) {
    return ((const __attribute__((address_space(4))) int32_t*)p.table)[(int64_t)t.b * p.ldt + (key >> p.c.page_shift)];
}
// Heads (rows of D entries) from the cache's start to the block's first key.
__device__ __forceinline__ int64_t attn_block(const AttnArgs& p, const AttnTile& t, int page, int key) {
    const uint32_t at = min((uint32_t)page, (uint32_t)p.c.pages - 1u);          // (below zero: past the end)
    return (int64_t)((uint64_t)at * (uint32_t)(p.c.heads << p.c.page_shift)) + ((t.g << p.c.page_shift) + (key & ((1 << p.c.page_shift) - 1)));
}
// Block `b` of the tile at `key`, or the last one that has keys.
__device__ __forceinline__ int block_key(const AttnTile& t, int key, int b) { return min(key + 16 * b, t.k1 - 1) & ~15; }

__device__ __forceinline__ float scale_of(uint8_t e) { return ldexpf(1.f, (int)e - 127); }

// Eight e4m3 values times a power of two.
__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// LDS tiles of keys, a row of 2 D bytes in 16-byte chunks.  K: 16 consecutive rows at one chunk index; V: transposing reads of eight rows
// by 32 bytes (lf_device.h): each must cover 256 bytes that are distinct modulo 256.
template <int D> __device__ __forceinline__ int k_off(int row, int chunk) {
    return row * (2 * D) + ((chunk ^ (D == 64 ? row >> 1 & 7 : row & 15)) << 4);
}
template <int D> __device__ __forceinline__ int v_off(int row, int chunk) {
    return row * (2 * D) + ((chunk ^ (D == 64 ? (row >> 1 & 3) << 1 : (row & 7) << 1)) << 4);
}
// V^T fragment of 16 entries by the 32 keys from row r0 on.
template <int D>
__device__ __forceinline__ bf16x8 v_frag(const char* v, int r0, int block) {
    const int l = threadIdx.x & 63, row = r0 + 4 * (l >> 4) + ((l & 15) >> 2), col = 16 * block + ((l & 3) << 2);
    const int off = v_off<D>(row, col >> 3) + ((col & 7) << 1);
    return join_tr(lds_read_tr(v, off), lds_read_tr(v, off + 16 * 2 * D));      // (16 rows further: the same swizzle)
}

// Largest of a lane's scores, in steps of two: number n of 2 KB (the last with one score).  Written as such: from fmaxf the compiler makes an
// instruction more for every score, to quiet NaNs.  It does not know the distance that the matrix pipe's results need before these
// read them: nine wait states stand before the first, or eight other instructions.
template <int KB>
__device__ __forceinline__ void top_step(float& top, const f32x4 (&s)[KB], int n) {
    const float x = s[n / 2][n % 2 * 2], y = s[n / 2][n % 2 * 2 + 1];
    if (n == 0) asm volatile("v_max_f32 %0, %1, %2" : "=v"(top) : "v"(x), "v"(y));
    else asm volatile("v_max3_f32 %0, %0, %1, %2" : "+v"(top) : "v"(x), "v"(y));
}
// The larger of this lane's and of that 16 (ROW; otherwise 32) lanes away.
template <bool ROW>
__device__ __forceinline__ void top_over_lanes(float& top) {
    const uint32_t x = __builtin_bit_cast(uint32_t, top);
    const auto both = ROW ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
    asm("v_max_f32 %0, %1, %2" : "=v"(top) : "v"((uint32_t)both[0]), "v"((uint32_t)both[1]));
}
template <int KB>
__device__ __forceinline__ float top_of(const f32x4 (&s)[KB]) {
    float top;
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 8");
#pragma unroll
    for (int n = 0; n < 2 * KB; ++n) top_step<KB>(top, s, n);
    top_over_lanes<true>(top);
    top_over_lanes<false>(top);
    return top;
}

// p = 2^(scale s - m).  m is the reference of the 16 queries of a block, the same in the four lanes of a query.  It follows the largest score only
// when that is more than 2^8 above it, so that most steps leave the sums as they are (p of up to 2^8 are as exact as those below
// 1).  Returns whether any has moved; back: what the sums are to be multiplied by.
// top: over the four lanes of a query.
template <int NQ>
__device__ __forceinline__ bool follow(const float (&top)[NQ], float (&m)[NQ], float (&back)[NQ], float scale) {
    bool rises = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) rises |= __builtin_fmaf(top[i], scale, -m[i]) > 8.f;
    if (!__any(rises)) return false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float to = __builtin_fmaf(top[i], scale, -m[i]) > 8.f ? top[i] * scale : m[i];
        back[i] = to == m[i] ? 1.f : __builtin_amdgcn_exp2f(m[i] - to);
        m[i] = to;
    }
    return true;
}
// References past kFar.  p_of takes the scaled score exactly, m is rounded: past 2^24 their difference is no longer near 0 for the largest score itself, and past 2^31
// its power of two is infinity or 0.  Such a row counts its scores from one of them (base: a float for every query of the wave, in LDS, read
// where far is set; zero for the other rows) and m from there on, so that the largest score's difference is exact.  Rare: a branch a step on a
// scalar, and nothing kept in registers (us, without / with: 278 / 278.5 for the chunks below, 343.9 / 344.9 over an fp8 cache, 61.3 / 62.5 for 16 x 6 tokens over
// up to 9000 keys, fp8, long single tokens level).
template <int NQ, int KB>
__device__ __forceinline__ void count_from_base(f32x4 (&s)[NQ][KB], float (&top)[NQ], const float* base, int c) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float d = base[16 * i + c];
        top[i] -= d;
#pragma unroll
        for (int b = 0; b < KB; ++b) s[i][b] -= d;
    }
}
// Behind follow(), where it has moved a reference.
template <int NQ, int KB>
__device__ __forceinline__ void move_base(f32x4 (&s)[NQ][KB], const float (&top)[NQ], float (&m)[NQ], float* base, int c, int& far) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < NQ; ++i) any |= fabsf(m[i]) > kFar && m[i] != kNone;
    if (__builtin_expect(!__any(any), 1)) return;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const bool moves = fabsf(m[i]) > kFar && m[i] != kNone;
        const float d = moves ? top[i] : 0.f;
        base[16 * i + c] = far ? base[16 * i + c] + d : d;           // (the four lanes of a query write the same)
        m[i] = moves ? 0.f : m[i];
#pragma unroll
        for (int b = 0; b < KB; ++b) s[i][b] -= d;
    }
    far = 1;
}
// The references as the other waves and parts know them, from 0.
template <int NQ>
__device__ __forceinline__ void count_from_zero(float (&m)[NQ], const float* base, int c, float scale) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) m[i] = __builtin_fmaf(base[16 * i + c], scale, m[i]);
}
__device__ __forceinline__ float p_of(float s, float scale, float m) { return __builtin_amdgcn_exp2f(__builtin_fmaf(s, scale, -m)); }

// The lane's number, formed where it is asked for: in code that runs rarely, or after a loop, so that nothing derived from it is kept through the loop.
__device__ __forceinline__ int lane_here() {
    int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(l));
    return l;
}

__device__ __forceinline__ bool sees(int pos, int key, int window) { return key <= pos && (!window || key > pos - window); }

// Hides from query `pos` what it may not see of the keys key0 + 16 b + 4 q + e.
template <int KB>
__device__ __forceinline__ void hide(f32x4 (&s)[KB], int key0, int pos, int window) {
    const int q4 = lane_here() >> 4 << 2;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!sees(pos, key0 + 16 * b + q4 + e, window)) s[b][e] = -__builtin_inff();
        }
}

// A lane's sum of the p that it holds: of the rounded ones, as the product takes them.
__device__ __forceinline__ float add_pair(uint32_t p2, float sum) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, p2), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
}

// O^T += V^T P^T over the 32 keys of a tile of values.  Fragments are read two ahead of their use.
template <int D, int NQ>
__device__ __forceinline__ void add_values(f32x4 (&o)[NQ][D / 16], const bf16x8 (&pf)[NQ], const char* v) {
    constexpr int DB = D / 16;
    bf16x8 vf[3];
    vf[0] = v_frag<D>(v, 0, 0);
    vf[1] = v_frag<D>(v, 0, 1);
#pragma unroll
    for (int n = 0; n < DB; ++n) {
        if (n + 2 < DB) vf[(n + 2) % 3] = v_frag<D>(v, 0, n + 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NQ; ++i) o[i][n] = LF_MFMA(vf[n % 3], pf[i], o[i][n]);
    }
}

// Tiles of which some rows see a part: 0 x infinity or NaN must not reach a row that does not see the key.  What is not finite is cleared on
// its way into LDS and, if there is any, read again and added key by key to the rows that see the key.
__device__ __forceinline__ u32x4 not_finite(u32x4 v) {       // 0xFFFF in the halves that are
    u32x4 m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = v[i] & 0x7FFF7FFFu;
        m[i] = ((x & 0xFFFFu) >= 0x7F80u ? 0xFFFFu : 0u) | (x >= 0x7F800000u ? 0xFFFF0000u : 0u);
    }
    return m;
}
template <int D, bool FP8, int NQ, int KB>
__device__ __forceinline__ void add_not_finite(const AttnArgs& p, const AttnTile& t, f32x4 (&o)[NQ][D / 16], const int (&pos)[NQ], int key0) {
    const int q = lane_here() >> 4;
#pragma unroll 1
    for (int k = 0; k < min(16 * KB, t.k1 - key0); ++k) {
        const int at16 = (key0 + k) & ~15;
        const int64_t at = attn_block(p, t, page_of(p, t, at16), at16) + (k & 15);
        const char* row = (const char*)p.c.v + at * (D * (FP8 ? 1 : 2)) + q * (FP8 ? 4 : 8);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            u32x2 x;
            if constexpr (FP8) {
                const uint32_t y = *(const uint32_t*)(row + 16 * d);
                x = __builtin_bit_cast(u32x4, widen8(y, y, scale_of(p.c.v_exp[at]))).xy;
            } else {
                x = *(const u32x2*)(row + 32 * d);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t y = e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16;
                const bool bad = (y & 0x7F800000u) == 0x7F800000u;
#pragma unroll
                for (int i = 0; i < NQ; ++i) o[i][d][e] += bad && sees(pos[i], key0 + k, p.window) ? __builtin_bit_cast(float, y) : 0.f;
            }
        }
    }
}

// Position of the token of row `row` (of the tile's sequence and head).
__device__ __forceinline__ int pos_of(const AttnArgs& p, const AttnTile& t, int row) { return t.kv - t.n + row / p.group; }
__device__ __forceinline__ const lora_bf16* q_row(const AttnArgs& p, const AttnTile& t, int row) {
    const int tok = row / p.group;
    return p.q + (int64_t)(t.first + tok) * p.ldq + (int64_t)(t.g * p.group + row - tok * p.group) * p.c.D;
}

// Token `tok` is one of more than there are keys: its row sees none and is zeros.  Every other row sees its own token's key: if all scores that it
// sees are -infinity its sum is 0 as well, and the result NaN, 0 / 0.
__device__ __forceinline__ bool sees_nothing(const AttnTile& t, int tok) { return t.kv - t.n + tok < 0; }

// Four entries from `d` on of a finished row: o = sum of p v, l = sum of p, m = their reference.
__device__ __forceinline__ void put(const AttnArgs& p, const AttnTile& t, int row, int d, f32x4 o, float m, float l) {
    const int tok = row / p.group, head = t.g * p.group + row - tok * p.group;
    if (t.parts > 1) {
        const int64_t at = (int64_t)t.split * p.T * p.H + (int64_t)(t.first + tok) * p.H + head;
        *(f32x4*)(p.part_o + at * p.c.D + d) = o;
        if (d == 0) {
            p.part_ml[2 * at] = m;
            p.part_ml[2 * at + 1] = l;
        }
        return;
    }
    const float inv = sees_nothing(t, tok) ? 0.f : 1.f / l;
    u32x2 v;
    v.x = pack_bf16x2(o[0] * inv, o[1] * inv);
    v.y = pack_bf16x2(o[2] * inv, o[3] * inv);
    *(u32x2*)(p.out + (int64_t)(t.first + tok) * p.ldo + (int64_t)head * p.c.D + d) = v;
}

// The fragments have come in: the waits for them stand here, not where they are used, in the loops, where they would be for whatever the loops have
// asked for in the meantime.
template <int N>
__device__ __forceinline__ void have(bf16x8 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

// ---- few rows --------------------------------------------------------------------------------------
// NQ blocks of 16 rows; a wave takes every fourth tile of 32 keys, and asks for the next tile's values before and its keys behind the scores of this
// one.  Measured (a read of 2 GiB: 6.0 TB/s): four sequences of 33000 - 131072 keys, bf16, 1.34 GB, 229 us, 5.9 TB/s; 32 of 200 - 4000, fp8, 139 MB, 32 us, 4.3 TB/s,
// some 6 us of it until the first keys are there (lengths, page numbers, keys: one after the other).  Two tiles of fp8 under way, with the registers that
// takes, 41 us for the latter launch and the join instead of 37.
template <int D, bool FP8, int NQ>
struct Few {
    static constexpr int KEYS = 32, WAVES = 4;
    static constexpr int KL = 2 * D / (FP8 ? 64 : 32);             // 16-byte loads of a lane for the keys of a tile
    static constexpr int VL = KEYS * D * (FP8 ? 1 : 2) / 1024;     // ... for the values
    static constexpr int V_BYTES = KEYS * D * 2, O_BYTES = 16 * NQ * D * 4;
    static constexpr int WAVE_LDS = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
    static constexpr int BASE = WAVES * WAVE_LDS + WAVES * NQ * 16 * 8, LDS = BASE + WAVES * NQ * 16 * 4;
};

template <int D, bool FP8, int NQ>
__global__ void __launch_bounds__(256, NQ == 1 ? 2 : 1) attn_few_kernel(AttnArgs p) {
    using C = Few<D, FP8, NQ>;
    constexpr int KK = D / 32, DB = D / 16;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    AttnTile t;
    if (!attn_tile<16 * NQ>(p, t)) return;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;
    char* mine = smem + w * C::WAVE_LDS;
    float* base = (float*)(smem + C::BASE) + w * NQ * 16;
    int far = 0;

    // queries: step kk holds entries 32 kk + 8 q .. + 7, fp8 64 (kk / 2) + 16 q + 8 (kk & 1) .. + 7 (as a 16-byte load of a key brings them)
    bf16x8 qf[NQ][KK];
    int pos[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int row = t.row0 + min(16 * i + c, t.rows - 1);
        pos[i] = pos_of(p, t, row);
        const lora_bf16* src = q_row(p, t, row);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
            qf[i][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(src + (FP8 ? 64 * (kk / 2) + 16 * q + 8 * (kk & 1) : 32 * kk + 8 * q)));
    }
    const int pos_lo = pos_of(p, t, t.row0);
#pragma unroll
    for (int i = 0; i < NQ; ++i) have(qf[i]);
    f32x4 o[NQ][DB];
    float m[NQ], sum[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        m[i] = kNone;
        sum[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kr[C::KL], vr[C::VL];
    uint8_t ke[2], ve[C::VL];
    const char *kc = (const char*)p.c.k, *vc = (const char*)p.c.v;
    constexpr int ESZ = FP8 ? 1 : 2, LANES = D * ESZ / 16;          // lanes to a row of values
    int pages[2];                                           // of the blocks of the tile that is asked for next
    int64_t blk[2];
    auto look_up = [&](int key) {
#pragma unroll
        for (int b = 0; b < 2; ++b) pages[b] = page_of(p, t, block_key(t, key, b));
    };
    auto find = [&](int key) {
#pragma unroll
        for (int b = 0; b < 2; ++b) blk[b] = attn_block(p, t, pages[b], block_key(t, key, b));
    };
    auto load_k = [&]() {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t at = blk[b] + c;
#pragma unroll
            for (int i = 0; i < C::KL / 2; ++i) kr[b * (C::KL / 2) + i] = *(const u32x4*)(kc + at * (D * ESZ) + 64 * i + 16 * q);
            if constexpr (FP8) ke[b] = p.c.k_exp[at];
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int i = 0; i < C::VL; ++i) {
            const int row = i * (64 / LANES) + l / LANES;
            const int64_t at = (row < 16 ? blk[0] : blk[1]) + (row & 15);
            vr[i] = *(const u32x4*)(vc + at * (D * ESZ) + l % LANES * 16);
            if constexpr (FP8) ve[i] = p.c.v_exp[at];
        }
    };

    constexpr int STEP = C::WAVES * C::KEYS;
    int key = t.k0 + C::KEYS * w;
    if (key < t.k1) {
        look_up(key);
        find(key);
        look_up(key + STEP);
        load_k();
        load_v();
    }
    for (; key < t.k1; key += STEP) {
        const bool more = key + STEP < t.k1;
        const bool whole = key + C::KEYS - 1 <= pos_lo && (!p.window || key > pos_of(p, t, t.row0 + t.rows - 1) - p.window);
        bool bad = false;                                    // a value that is not finite, where that matters
        // values to LDS; a row past the end holds anything, and 0 x anything need not be 0
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < C::VL; ++i) {
            const int row = i * (64 / LANES) + l / LANES, ch = l % LANES;
            const bool in = key + row < t.k1;
            u32x4 lo = vr[i], hi;
            if constexpr (FP8) {
                const float sc = scale_of(ve[i]);
                lo = __builtin_bit_cast(u32x4, widen8(vr[i][0], vr[i][1], sc));
                hi = __builtin_bit_cast(u32x4, widen8(vr[i][2], vr[i][3], sc));
            }
            if (!whole) {
                lo = in ? lo : u32x4{0u, 0u, 0u, 0u};
                u32x4 m = not_finite(lo);
                lo &= ~m;
                if constexpr (FP8) {
                    hi = in ? hi : u32x4{0u, 0u, 0u, 0u};
                    const u32x4 mh = not_finite(hi);
                    hi &= ~mh;
                    m |= mh;
                }
                bad |= (m[0] | m[1] | m[2] | m[3]) != 0;
            }
            if constexpr (FP8) {
                *(u32x4*)(mine + v_off<D>(row, 2 * ch)) = lo;
                *(u32x4*)(mine + v_off<D>(row, 2 * ch + 1)) = hi;
            } else {
                *(u32x4*)(mine + v_off<D>(row, ch)) = lo;
            }
        }
        if (more) {
            find(key + STEP);
            look_up(key + 2 * STEP);
            load_v();
        }
        f32x4 s[NQ][2];
#pragma unroll
        for (int i = 0; i < NQ; ++i) s[i][0] = s[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                bf16x8 kf;
                if constexpr (FP8) {
                    const u32x4 r = kr[b * (C::KL / 2) + kk / 2];
                    kf = kk & 1 ? widen8(r[2], r[3], scale_of(ke[b])) : widen8(r[0], r[1], scale_of(ke[b]));
                } else {
                    kf = __builtin_bit_cast(bf16x8, kr[b * (C::KL / 2) + kk]);
                }
#pragma unroll
                for (int i = 0; i < NQ; ++i) s[i][b] = LF_MFMA(kf, qf[i][kk], s[i][b]);
            }
        if (more) load_k();
        float top[NQ], back[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (!whole) hide(s[i], key, pos[i], p.window);
            top[i] = top_of<2>(s[i]);
        }
        if (__builtin_expect(far, 0)) count_from_base(s, top, base, lane_here() & 15);
        if (follow<NQ>(top, m, back, p.scale)) {
            move_base(s, top, m, base, lane_here() & 15, far);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                sum[i] *= back[i];
#pragma unroll
                for (int d = 0; d < DB; ++d) o[i][d] *= back[i];
            }
        }
        bf16x8 pf[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            u32x4 pw;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4& x = s[i][j / 2];
                pw[j] = pack_bf16x2(p_of(x[j % 2 * 2], p.scale, m[i]), p_of(x[j % 2 * 2 + 1], p.scale, m[i]));
                sum[i] = add_pair(pw[j], sum[i]);
            }
            pf[i] = __builtin_bit_cast(bf16x8, pw);
        }
        asm volatile("" ::: "memory");
        add_values<D, NQ>(o, pf, mine);
        if (__any(bad)) add_not_finite<D, FP8, NQ, 2>(p, t, o, pos, key);
    }

    // the four waves' sums, brought to one reference
    if (far) count_from_zero(m, base, c, p.scale);
    float* ml = (float*)(smem + C::WAVES * C::WAVE_LDS);              // [row][wave] of m, then of l
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        sum[i] = over_quarters(sum[i], [](float a, float b) { return a + b; });
        if (q == 0) {
            ml[(16 * i + c) * C::WAVES + w] = m[i];
            ml[(NQ * 16 + 16 * i + c) * C::WAVES + w] = sum[i];
        }
    }
    __syncthreads();
    const auto joined = [&](int row, float& top, float& l) {
        const f32x4 a = *(const f32x4*)(ml + row * C::WAVES), b = *(const f32x4*)(ml + (NQ * 16 + row) * C::WAVES);
        top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) l += b[i] * __builtin_amdgcn_exp2f(a[i] - top);
    };
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        float top, l;
        joined(16 * i + c, top, l);
        const float f = __builtin_amdgcn_exp2f(m[i] - top);
#pragma unroll
        for (int d = 0; d < DB; ++d) *(f32x4*)(mine + ((16 * i + c) * D + (((4 * d + q) ^ c) << 2)) * 4) = o[i][d] * f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.rows * (D / 4); i += 256) {
        const int row = i / (D / 4), ch = i % (D / 4);
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < C::WAVES; ++k) v += *(const f32x4*)(smem + k * C::WAVE_LDS + (row * D + ((ch ^ (row & 15)) << 2)) * 4);
        float top, l;
        joined(row, top, l);
        put(p, t, t.row0 + row, 4 * ch, v, top, l);
    }
}

// f(0), f(1), .., f(N - 1), each with its number as a constant.
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}
// How many of `items`, spread over `slots`, come before slot n.
constexpr int slots_before(int n, int items, int slots) { return n <= 0 ? 0 : n >= slots ? items : (n * items + slots - 1) / slots; }

// ---- many rows --------------------------------------------------------------------------------------
// Two workgroups of four waves on a compute unit, 32 rows to a wave, so that what is read of a tile in LDS serves two blocks of rows.  The scores of
// tile n + 1, the softmax of tile n and the values of tile n - 1 are one stream of instructions, in which the vector ones stand between the matrix
// ones, two to each: only those of the same wave run beside a matrix instruction, those of other waves wait for it.  Measured: two
// prompts' 1021 new tokens over 5003 and 16000 keys, 32 heads of 128 to 8, 250 GFLOP, 265 us, 940 TFLOP/s (a product of 8192^3: 1320); bound by the issue of
// instructions (a step of 64 keys takes 3300 cycles, of which its 64 matrix instructions and the 64 of the SIMD's other wave 2050).
template <int D, bool FP8>
struct Many {
    static constexpr int KEYS = 64, ROWS = 128, NQ = 2;
    // two tiles of keys, two of values; flags; of every row the score that it counts from; fp8 a tile as it is held
    static constexpr int TILE = KEYS * D * 2, FLAGS = 4 * TILE, BASE = FLAGS + 16, RAW = BASE + ROWS * 4;
    static constexpr int LDS = RAW + (FP8 ? KEYS * D : 0);
};

// Copy I of a block of 16 keys (or values) into LDS, 1 KB: the instruction's offset, the same for memory and LDS, counts from the middle.  The first
// sets M0 for the others.
template <int D, bool KEYS, int I>
__device__ __forceinline__ void copy_one(const char* from, uint32_t lane, uint32_t m0) {
    constexpr int NP = D / 32, RPC = 512 / D;
    const uint32_t swz = (KEYS ? k_off<D>(RPC * I, 0) : v_off<D>(RPC * I, 0)) & (2 * D - 1);
    copy16_to_lds<pass_imm(NP, I), I == 0>(from + NP / 2 * 1024, lane ^ swz, m0);
}
template <int D, bool KEYS, int I = 0>
__device__ __forceinline__ void copy_block(const char* from, uint32_t lane, uint32_t m0) {
    if constexpr (I < D / 32) {
        copy_one<D, KEYS, I>(from, lane, m0);
        copy_block<D, KEYS, I + 1>(from, lane, m0);
    }
}

template <int NR, int I = 0>
__device__ __forceinline__ void copy_raw(const char* from, uint32_t lane, uint32_t m0) {
    if constexpr (I < NR) {
        copy16_to_lds<I * 1024, I == 0>(from, lane, m0);
        copy_raw<NR, I + 1>(from, lane, m0);
    }
}

template <int D, bool FP8>
__global__ void __launch_bounds__(256, 2) attn_many_kernel(AttnArgs p) {
    using C = Many<D, FP8>;
    constexpr int NQ = C::NQ, KK = D / 32, DB = D / 16, KB = C::KEYS / 16;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    AttnTile t;
    if (!attn_tile<C::ROWS>(p, t)) return;
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = l & 15, q = l >> 4;

    bf16x8 qf[NQ][KK];
    int pos[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const int row = t.row0 + min(32 * w + 16 * i + c, t.rows - 1);
        pos[i] = pos_of(p, t, row);
        const lora_bf16* src = q_row(p, t, row);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qf[i][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(src + 32 * kk + 8 * q));
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) have(qf[i]);
    const int pos_lo = pos_of(p, t, t.row0 + min(32 * w, t.rows - 1)), pos_hi = pos_of(p, t, t.row0 + min(32 * w + 31, t.rows - 1));
    f32x4 o[NQ][DB];
    float m[NQ], sum[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        m[i] = kNone;
        sum[i] = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Straight into LDS, wave w the 16 keys of block w, which lie side by side in their page; a lane's source chosen so that what it writes lies
    // swizzled.  fp8: as it is, into a place of the wave's own, from where the wave widens it into the tile.
    constexpr int RPC = 512 / D;                             // bf16: rows of a 1 KB copy
    const uint32_t lds = lds_addr_of(smem);
    // source of a lane in copy 0; in copy i, 1 KB further, only the swizzle differs, by a constant: k_off, v_off of row RPC * i
    auto lane_source = [&](bool keys) {
        const int le = lane_here(), row = le / (D / 8);
        return (uint32_t)((row * 2 * D + le % (D / 8) * 16) ^ ((keys ? k_off<D>(row, 0) : v_off<D>(row, 0)) & (2 * D - 1)));
    };
    constexpr int NR = FP8 ? D / 64 : 1, RPR = 1024 / D;     // fp8: copies of a block, rows of one
    uint8_t ex[NR];                                         // ... and of this lane's row of each the exponent
    // first head entry of the wave's block in the tiles whose values (at_v) and keys (at_k) are asked for next, and in the one between; page of the
    // one after
    int64_t at_v, at_n, at_k;
    int page_after;
    auto page_at = [&](int key) { return page_of(p, t, block_key(t, key, w)); };
    auto block_at = [&](int page, int key) { return attn_block(p, t, page, block_key(t, key, w)); };
    auto source = [&](bool keys, int64_t at) { return (const char*)(keys ? p.c.k : p.c.v) + at * (FP8 ? D : 2 * D); };
    // keys (values) into half `stage` of their part of LDS
    auto bring = [&](bool keys, int64_t at, int stage) {
        const char* from = source(keys, at);
        if constexpr (FP8) {
            copy_raw<NR>(from, lane_here() * 16, __builtin_amdgcn_readfirstlane(lds + C::RAW + w * 16 * D));
#pragma unroll
            for (int i = 0; i < NR; ++i) ex[i] = (keys ? p.c.k_exp : p.c.v_exp)[at + i * RPR + lane_here() / (D / 16)];
        } else {
            const uint32_t m0 = __builtin_amdgcn_readfirstlane(lds + (keys ? 0 : 2 * C::TILE) + stage * C::TILE + w * 32 * D + D / 64 * 1024);
            if (keys) copy_block<D, true>(from, lane_source(true), m0);
            else copy_block<D, false>(from, lane_source(false), m0);
        }
    };
    // fp8: row and first chunk in the tile of 16 bytes of copy i, and what they are widened to
    struct Wide { int row, chunk; u32x4 lo, hi; };
    auto widened = [&](int i) {
        const int le = lane_here();
        const u32x4 raw = *(const u32x4*)(smem + C::RAW + w * 16 * D + i * 1024 + le * 16);
        const float sc = scale_of(ex[i]);
        return Wide{16 * w + i * RPR + le / (D / 16), le % (D / 16) * 2, __builtin_bit_cast(u32x4, widen8(raw[0], raw[1], sc)),
                    __builtin_bit_cast(u32x4, widen8(raw[2], raw[3], sc))};
    };
    auto brought_k = [&](int stage) {
        wait_slab_loads();
        if constexpr (FP8)
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const Wide x = widened(i);
                *(u32x4*)(smem + stage * C::TILE + k_off<D>(x.row, x.chunk)) = x.lo;
                *(u32x4*)(smem + stage * C::TILE + k_off<D>(x.row, x.chunk + 1)) = x.hi;
            }
    };
    // flag of a stage: the number of its tile if a value in it is not finite, where that matters (a tile that not all rows see in whole)
    const int first_pos = pos_of(p, t, t.row0), last_pos = pos_of(p, t, t.row0 + t.rows - 1);
    auto all_whole = [&](int key) { return key + C::KEYS - 1 <= first_pos && (!p.window || key > last_pos - p.window); };
    int* flags = (int*)(smem + C::FLAGS);
    float* base = (float*)(smem + C::BASE) + 32 * w;
    int far = 0;
    auto brought_v = [&](int key, int stage) {
        char* st = smem + 2 * C::TILE + stage * C::TILE;
        const bool guard = !all_whole(key);
        bool bad = false;
        // a row past the end holds anything, and 0 x anything need not be 0
        auto guarded = [&](u32x4 x, int row) {
            if (key + row >= t.k1) x = u32x4{0u, 0u, 0u, 0u};
            const u32x4 m = not_finite(x);
            bad |= (m[0] | m[1] | m[2] | m[3]) != 0;
            return x & ~m;
        };
        wait_slab_loads();
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                Wide x = widened(i);
                if (guard) {
                    x.lo = guarded(x.lo, x.row);
                    x.hi = guarded(x.hi, x.row);
                }
                *(u32x4*)(st + v_off<D>(x.row, x.chunk)) = x.lo;
                *(u32x4*)(st + v_off<D>(x.row, x.chunk + 1)) = x.hi;
            }
        } else if (guard) {
            for (int i = lane_here(); i < 2 * D; i += 64) {  // the wave's own 16 rows, chunk by chunk
                u32x4* at = (u32x4*)(st + w * 32 * D + i * 16);
                *at = guarded(*at, 16 * w + i / (D / 8));
            }
        }
        if (__any(bad) && lane_here() == 0) flags[stage] = key;
    };

    // Step n forms the scores of tile n + 1 and adds the values of tile n - 1, while between these matrix instructions the exponentials of tile n
    // and then the maxima of tile n + 1 run: the vector unit can work beside the matrix pipe only between the matrix instructions
    // of the same wave (two to three instructions to each; those of another wave of the SIMD wait), so every one gets its share.
    constexpr int AHEAD = 2, FK = KB * KK, FV = KB / 2 * DB;       // fragments on their way from LDS; fragments of a tile
    constexpr int NS = FK * NQ, NV = FV * NQ;                      // matrix instructions of the scores and of the values
    constexpr int EXPS = 4 * KB * NQ, EXP_SLOTS = NS, TOPS = 2 * KB * NQ, TOP_FROM = NS + NV / 3, TOP_SLOTS = NV / 3;
    constexpr int LANES_FROM = TOP_FROM + TOP_SLOTS, LANES_SLOTS = NS + NV - LANES_FROM;
    bf16x8 fr[AHEAD + 1];
    const char *kst, *vst;
    auto read_k = [&](int f) {
        if (f < FK) fr[f % (AHEAD + 1)] = __builtin_bit_cast(bf16x8, *(const u32x4*)(kst + k_off<D>(16 * (f / KK) + c, 4 * (f % KK) + q)));
    };
    auto read_v = [&](int f) {
        if (f < FV) fr[(FK + f) % (AHEAD + 1)] = v_frag<D>(vst, 32 * (f / DB), f % DB);
    };
    struct Weights { uint32_t w[NQ][KB / 2][4]; };          // P of a tile, two to a word
    f32x4 sa[NQ][KB], sb[NQ][KB];                           // scores and weights of this tile and its neighbour, in turn
    Weights wa, wb;
    float top[NQ], add[NQ];                                 // of the next tile's scores; sums of this tile's weights
    auto weigh = [&](f32x4 (&s)[NQ][KB], Weights& pw, int n) {
        const int i = n / (4 * KB), b = n / 4 % KB, e = n & 3;
        f32x4& x = s[i][b];
        x[e] = p_of(x[e], p.scale, m[i]);
        if (e & 1) {
            uint32_t& two = pw.w[i][b / 2][2 * (b & 1) + e / 2];
            two = pack_bf16x2(x[e - 1], x[e]);
            add[i] = add_pair(two, add[i]);
        }
    };
    auto pfrag = [&](const Weights& pw, int i, int h) { return __builtin_bit_cast(bf16x8, u32x4{pw.w[i][h][0], pw.w[i][h][1], pw.w[i][h][2], pw.w[i][h][3]}); };
    auto score = [&](f32x4 (&next)[NQ][KB], int n) {        // matrix instruction n of the scores
        const int f = n / NQ, b = f / KK, i = n % NQ;
        if (f % KK == 0) next[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
        next[i][b] = LF_MFMA(fr[f % (AHEAD + 1)], qf[i][f % KK], next[i][b]);
    };
    auto value = [&](const Weights& pw, int n) {            // ... of the values
        const int f = n / NQ, i = n % NQ;
        if (i == 0) read_v(f + AHEAD);
        o[i][f % DB] = LF_MFMA(fr[(FK + f) % (AHEAD + 1)], pfrag(pw, i, f / DB), o[i][f % DB]);
    };

    if (threadIdx.x < 2) flags[threadIdx.x] = -1;
    // what step 0 takes for the values of a tile before it
    for (int i = threadIdx.x; i < C::TILE / 16; i += 256) *(u32x4*)(smem + 3 * C::TILE + i * 16) = u32x4{0u, 0u, 0u, 0u};
    if (t.k0 < t.k1) {
        at_v = block_at(page_at(t.k0), t.k0);
        at_n = block_at(page_at(t.k0 + C::KEYS), t.k0 + C::KEYS);
        at_k = block_at(page_at(t.k0 + 2 * C::KEYS), t.k0 + 2 * C::KEYS);
        page_after = page_at(t.k0 + 3 * C::KEYS);
        bring(true, at_v, 0);
        brought_k(0);
        bring(true, at_n, 1);
        brought_k(1);
    }
    __syncthreads();
    // the first tile's scores by themselves
    kst = smem;
    if (t.k0 < t.k1) {
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) read_k(f);
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            if (n % NQ == 0) read_k(n / NQ + AHEAD);
            score(sa, n);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) top[i] = top_of<KB>(sa[i]);
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int h = 0; h < KB / 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) wb.w[i][h][j] = 0u;
    }
    __syncthreads();
    auto step = [&](f32x4 (&s)[NQ][KB], f32x4 (&next)[NQ][KB], Weights& pw, const Weights& before, int key, int stage) {
        // keys of tile n + 2 to where those of tile n were, values of tile n to where those of tile n - 2 were; bf16: copy by copy between the
        // matrix instructions, since a copy holds the wave up until the memory pipeline takes it
        constexpr int NP = D / 32, EVERY = 2;
        const char *from_k = nullptr, *from_v = nullptr;
        uint32_t lane_k = 0, lane_v = 0, m0_k = 0, m0_v = 0;
        const int64_t at_v_now = at_v;
        if constexpr (FP8) {
            bring(true, at_k, stage);
        } else {
            from_k = source(true, at_k);
            from_v = source(false, at_v);
            m0_k = __builtin_amdgcn_readfirstlane(lds + stage * C::TILE + w * 32 * D + D / 64 * 1024);
            m0_v = m0_k + 2 * C::TILE;
            lane_k = lane_source(true);
            lane_v = lane_source(false);
        }
        kst = smem + (stage ^ 1) * C::TILE;
        vst = smem + 2 * C::TILE + (stage ^ 1) * C::TILE;
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) read_k(f);
        const bool whole = key + C::KEYS - 1 <= pos_lo && (!p.window || key > pos_hi - p.window);
        float back[NQ];
        if (!whole)
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                hide(s[i], key, pos[i], p.window);
                top[i] = top_of<KB>(s[i]);
            }
        if (__builtin_expect(far, 0)) count_from_base(s, top, base, lane_here() & 15);
        const bool moved = follow<NQ>(top, m, back, p.scale);
        if (moved) move_base(s, top, m, base, lane_here() & 15, far);
#pragma unroll
        for (int i = 0; i < NQ; ++i) add[i] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
        each<NS + NV>([&](auto slot) {
            constexpr int n = slot();
            if constexpr (n < NS) {
                if constexpr (n % NQ == 0) {
                    read_k(n / NQ + AHEAD);
                    if constexpr (n / NQ + AHEAD >= FK) read_v(n / NQ + AHEAD - FK);
                }
                score(next, n);
            } else {
                value(before, n - NS);
            }
            constexpr int e0 = slots_before(n, EXPS, EXP_SLOTS), e1 = slots_before(n + 1, EXPS, EXP_SLOTS);
            each<e1 - e0>([&](auto k) { weigh(s, pw, e0 + k()); });
            constexpr int t0 = slots_before(n - TOP_FROM, TOPS, TOP_SLOTS), t1 = slots_before(n + 1 - TOP_FROM, TOPS, TOP_SLOTS);
            each<t1 - t0>([&](auto k) { top_step<KB>(top[(t0 + k()) / (2 * KB)], next[(t0 + k()) / (2 * KB)], (t0 + k()) % (2 * KB)); });
            constexpr int l0 = slots_before(n - LANES_FROM, 2 * NQ, LANES_SLOTS), l1 = slots_before(n + 1 - LANES_FROM, 2 * NQ, LANES_SLOTS);
            each<l1 - l0>([&](auto k) { top_over_lanes<(l0 + k()) / NQ == 0>(top[(l0 + k()) % NQ]); });
            if constexpr (n == NS + 2) {                    // where the next tiles lie
                at_v = at_n;
                at_n = at_k;
                at_k = block_at(page_after, key + 3 * C::KEYS);
                page_after = page_at(key + 4 * C::KEYS);
            }
            if constexpr (!FP8 && n % EVERY == EVERY - 1 && n / EVERY < 2 * NP) {
                constexpr int j = n / EVERY;
                if constexpr (j < NP) copy_one<D, true, j>(from_k, lane_k, m0_k);
                else copy_one<D, false, j - NP>(from_v, lane_v, m0_v);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (FP8 && n == NS - 1) {             // (one place for what is to be widened)
                brought_k(stage);
                bring(false, at_v_now, stage);
            }
        });
        if (key > t.k0 && !all_whole(key - C::KEYS) && flags[stage ^ 1] == key - C::KEYS)
            add_not_finite<D, FP8, NQ, KB>(p, t, o, pos, key - C::KEYS);
        if (moved) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                sum[i] *= back[i];
#pragma unroll
                for (int d = 0; d < DB; ++d) o[i][d] *= back[i];
            }
        }
#pragma unroll
        for (int i = 0; i < NQ; ++i) sum[i] += add[i];
        brought_v(key, stage);
        __syncthreads();
    };
    // (an even number of tiles: only the last part of a range can have an odd one, and no row sees keys past its end)
    int key = t.k0;
    for (; key < t.k1; key += 2 * C::KEYS) {
        step(sa, sb, wa, wb, key, 0);
        step(sb, sa, wb, wa, key + C::KEYS, 1);
    }
    if (t.k0 < t.k1) {
        vst = smem + 3 * C::TILE;
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) read_v(f);
#pragma unroll
        for (int n = 0; n < NV; ++n) value(wb, n);
        if (flags[1] == key - C::KEYS) add_not_finite<D, FP8, NQ, KB>(p, t, o, pos, key - C::KEYS);
    }
    if (far) count_from_zero(m, base, lane_here() & 15, p.scale);
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float total = over_quarters(sum[i], [](float a, float b) { return a + b; });
        const int le = lane_here(), row = 32 * w + 16 * i + (le & 15);
        if (row < t.rows)
#pragma unroll
            for (int d = 0; d < DB; ++d) put(p, t, t.row0 + row, 16 * d + 4 * (le >> 4), o[i][d], m[i], total);
    }
}

// ---- the parts' results, joined ---------------------------------------------------------------------
// D / 4 lanes read a row of a part, four entries each; running maximum and sum as in the kernels, four parts a step.  Many rows: each of these groups of lanes
// (8 of a workgroup, D = 64: 16) has a row of its own and goes through its parts.  Few rows, of perhaps many parts: a workgroup for a row, the parts shared
// out over the groups, whose results are joined in a fixed order.  Bound by the reading of the parts, which are in the memory-side cache: 2042 tokens of 32 heads in
// up to four parts, 134 MB, 16.5 us (a wave for a row, its maxima read first: 35); four tokens of 32 heads in 64 parts 5.5 us (with 7.8).
template <int D, int BM>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs p) {
    constexpr int LANES = D / 4, SLOTS = 256 / LANES, U = 4;
    constexpr bool SPREAD = BM < 128;
    constexpr int STEP = SPREAD ? SLOTS : 1;
    const int slot = threadIdx.x / LANES, d = threadIdx.x % LANES * 4;
    AttnTile t;
    const int per = (int)gridDim.x / (p.c.heads * p.B);     // workgroups for a head of a sequence
    int id = blockIdx.x;
    const int row0 = id % per * (SPREAD ? 1 : SLOTS), row = SPREAD ? row0 : row0 + slot;
    id /= per;
    t.g = id % p.c.heads;
    t.b = id / p.c.heads;
    t.tile = row0 / BM;
    if (!attn_rows<BM>(p, t) || t.parts == 1 || row - t.row0 >= t.rows) return;
    const int tok = row / p.group, head = t.g * p.group + row - tok * p.group;
    const int64_t at = (int64_t)(t.first + tok) * p.H + head, plane = (int64_t)p.T * p.H;
    float m = kNone, sum = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = SPREAD ? slot : 0; i0 < t.parts; i0 += U * STEP) {
        f32x4 v[U];
        float pm[U], pl[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * STEP;
            pm[u] = kNone;
            pl[u] = 0.f;
            v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (i < t.parts) {
                const float* ml = p.part_ml + 2 * (i * plane + at);
                pm[u] = ml[0];
                pl[u] = ml[1];
                v[u] = *(const f32x4*)(p.part_o + (i * plane + at) * D + d);
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) top = fmaxf(top, pm[u]);
        const float back = __builtin_amdgcn_exp2f(m - top);
        o *= back;
        sum *= back;
        m = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = __builtin_amdgcn_exp2f(pm[u] - top);
            o += v[u] * f;
            sum += pl[u] * f;
        }
    }
    if constexpr (SPREAD) {
        __shared__ f32x4 red_o[SLOTS][LANES];
        __shared__ float red_ml[SLOTS][2];
        red_o[slot][d / 4] = o;
        if (d == 0) {
            red_ml[slot][0] = m;
            red_ml[slot][1] = sum;
        }
        __syncthreads();
        if (slot) return;
        const int n = min(SLOTS, t.parts);
        for (int i = 1; i < n; ++i) m = fmaxf(m, red_ml[i][0]);
        o = f32x4{0.f, 0.f, 0.f, 0.f};
        sum = 0.f;
        for (int i = 0; i < n; ++i) {
            const float f = __builtin_amdgcn_exp2f(red_ml[i][0] - m);
            o += red_o[i][d / 4] * f;
            sum += red_ml[i][1] * f;
        }
    }
    const float inv = sees_nothing(t, tok) ? 0.f : 1.f / sum;
    *(u32x2*)(p.out + (int64_t)(t.first + tok) * p.ldo + (int64_t)head * D + d) =
        u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
}

// ---- launches ---------------------------------------------------------------------------------------
// The most keys that a tile sees.
static int64_t keys_of_tile(int rows, int group, int64_t max_kv, int window) {
    return window ? std::min<int64_t>(max_kv, (int64_t)window + (rows + group - 1) / group + 16) : max_kv;
}
// Parts of a range (plan_attn): as many as make per_unit workgroups to a compute unit, of `least` keys and more, at most `most`; `one`: for one sequence (many
// rows: for a batch too), otherwise for a batch.
struct PartsRule { bool few, one; int per_unit, least, most; };
constexpr PartsRule kParts[] = {{true, true, 2, 512, 1 << 30}, {true, false, 4, 512, 1 << 30}, {true, false, 8, 2048, 1 << 30},
                                {false, true, 1, 256, 1 << 30}, {false, true, 2, 1024, 1 << 30}, {false, false, 8, 1536, 16}};

// Rows of partial results (parts x T x H) that no step of at most these sizes exceeds, though a smaller one is cut into more parts.  Of T <= B * max_new tokens in
// `tiles` of so many rows a sequence, c workgroups to a compute unit make c * kComputeUnits / (tiles * B * G) parts or fewer: parts x T x H is at most c * kComputeUnits
// rows times those of a sequence (few rows) or of a tile (many), and at most T x H times the parts that one sequence and one tile have.
int64_t attn_part_rows(int64_t T, int B, int G, int group, int max_new, int64_t max_kv, int window) {
    int64_t rows = 0;
    for (const PartsRule& u : kParts) {
        if (u.few ? group > 32 : (int64_t)max_new * group <= 32) continue;
        if (B == 1 && !u.one) continue;
        const int64_t units = (int64_t)u.per_unit * kComputeUnits;
        const int64_t of_seq = u.few ? std::min<int64_t>((int64_t)max_new * group, 32) / group * group : 128;
        const int64_t parts = std::min<int64_t>({units / G, keys_of_tile(u.few ? 32 : 128, group, max_kv, window) / u.least, u.most});
        if (parts > 1) rows = std::max(rows, std::min(units * of_seq, parts * T * G * group));
    }
    return rows;
}

AttnPlan plan_attn(int B, int G, int group, int D, int max_new, int64_t max_kv, int window) {
    AttnPlan pl;
    const int64_t rows = (int64_t)max_new * group;
    pl.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 128;
    const int64_t tiles = (rows + pl.rows - 1) / pl.rows;
    const int64_t keys = keys_of_tile(pl.rows, group, max_kv, window);
    // Parts, until there are so many workgroups to a compute unit, of so many keys and more.  Sequences differ in length, which only the device knows, so
    // that a batch of long ones takes more.  Few rows: one sequence 2, of 512; a batch 4, and 8 of 2048.  Many rows, whose parts' results cost 1 KB a row
    // (D = 128) to write and read again: one, of 256; 2, of 1024; a batch 8, of 1536, up to 16 parts.  us, this rule / others: few rows, four sequences of 33000 - 131072
    // keys 236 / 253 (4 to a compute unit), eight of 3000 - 65536 210 / 235 (4), 32 of 200 - 4000 36.9 / 37.8 (8, of 512), 128 of 500 - 3000 173 / 179 (8, of 512), one
    // of 131072 56 / 62 (4); many rows, two of 5003 and 16000, 1021 new 283 / 319 (4), four of 600 - 6000, 300 new 116 / 132 (of 4096), eight of 1000 - 2048, 512
    // new 144 / 207 (of 1024), 16 of 100 - 1000, 64 new 39 / 43 (2, of 512), one of 8192, 1024 new 148 / 154 (4, of 2048), two of 2000 - 3000, 60 new, D = 64
    // 18 / 19 (of 512), four of 12000 - 61000, 47 new 172 / 178 (39 parts).
    const int64_t have = std::max<int64_t>(tiles * B * G, 1);
    const auto up_to = [&](int per_unit, int64_t least) { return std::min<int64_t>(per_unit * kComputeUnits / have, keys / least); };
    int64_t parts = 1;
    for (const PartsRule& u : kParts)
        if (u.few == (pl.rows < 128) && (u.one ? B == 1 || !u.few : B > 1)) parts = std::max(parts, std::min<int64_t>(up_to(u.per_unit, u.least), u.most));
    const int64_t step = 128;
    pl.split_keys = (int)(((keys + parts - 1) / parts + step - 1) / step * step);
    if (pl.split_keys < step) pl.split_keys = step;
    pl.splits = (int)std::max<int64_t>(1, (keys + pl.split_keys - 1) / pl.split_keys);
    if (pl.splits == 1) pl.split_keys = 1 << 30;
    return pl;
}

template <auto KERNEL>
static hipError_t launch_lds(int lds, unsigned blocks, const AttnArgs& a, hipStream_t st) {
    static std::atomic<uint64_t> allowed{0};       // one per kernel
    const hipError_t e = allow_lds((const void*)KERNEL, lds, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(KERNEL, dim3(blocks), dim3(256), lds, st, a);
    return hipGetLastError();
}

template <int D, bool FP8>
static hipError_t launch_attn_t(const AttnArgs& a, int rows, unsigned blocks, hipStream_t st) {
    if (rows == 16) return launch_lds<attn_few_kernel<D, FP8, 1>>(Few<D, FP8, 1>::LDS, blocks, a, st);
    if (rows == 32) return launch_lds<attn_few_kernel<D, FP8, 2>>(Few<D, FP8, 2>::LDS, blocks, a, st);
    return launch_lds<attn_many_kernel<D, FP8>>(Many<D, FP8>::LDS, blocks, a, st);
}

template <int D>
static hipError_t launch_join(const AttnArgs& a, int rows, int max_new, hipStream_t st) {
    const int64_t all = (int64_t)max_new * a.group, slots = rows < 128 ? 1 : 1024 / D;
    const int64_t blocks = (all + slots - 1) / slots * a.c.heads * a.B;
    if (rows == 16) hipLaunchKernelGGL((attn_join_kernel<D, 16>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    else if (rows == 32) hipLaunchKernelGGL((attn_join_kernel<D, 32>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_join_kernel<D, 128>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_attn(AttnArgs a, const AttnPlan& p, int max_new, hipStream_t st) {
    a.tiles = (int)(((int64_t)max_new * a.group + p.rows - 1) / p.rows);
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    const unsigned blocks = (unsigned)((int64_t)a.tiles * a.splits * a.B * a.c.heads);
    hipError_t e;
    if (a.c.D == 64) e = a.c.fp8 ? launch_attn_t<64, true>(a, p.rows, blocks, st) : launch_attn_t<64, false>(a, p.rows, blocks, st);
    else e = a.c.fp8 ? launch_attn_t<128, true>(a, p.rows, blocks, st) : launch_attn_t<128, false>(a, p.rows, blocks, st);
    if (e != hipSuccess || a.splits == 1) return e;
    return a.c.D == 64 ? launch_join<64>(a, p.rows, max_new, st) : launch_join<128>(a, p.rows, max_new, st);
}

}  // namespace lf
