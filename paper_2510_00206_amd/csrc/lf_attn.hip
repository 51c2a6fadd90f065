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

#include "lf_gemm_parts.h"
#include "lf_serve.h"

namespace lf {

constexpr float kNone = -__builtin_inff();

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
    // Key/value heads of a sequence fastest, then sequences: with eight heads the tiles and parts that share keys are on one XCD.  Last tiles
    // first: they see the most keys.
    int id = blockIdx.x;
    t.g = id % p.c.heads;
    id /= p.c.heads;
    t.b = id % p.B;
    id /= p.B;
    t.split = id % p.splits;
    t.tile = p.tiles - 1 - id / p.splits;
    if (!attn_rows<BM>(p, t) || t.split >= t.parts) return false;
    t.k0 = t.key_lo + t.split * p.split_keys;
    t.k1 = t.split + 1 == p.splits ? t.key_hi : min(t.key_hi, t.k0 + p.split_keys);     // (the last takes what there is: lengths past max_kv)
    return true;
}

// Element offset of the first key of a 16-key block (in one page) of head g, in units of a head's entries; key < kv.
__device__ __forceinline__ int64_t attn_block(const AttnArgs& p, const AttnTile& t, int key) {
    int64_t page = p.table[(int64_t)t.b * p.ldt + (key >> p.c.page_shift)];
    page = page < 0 ? 0 : page >= p.c.pages ? p.c.pages - 1 : page;
    return ((page * p.c.heads + t.g) << p.c.page_shift) + (key & ((1 << p.c.page_shift) - 1));
}

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

// Running maximum and sum of the 16 queries of a block; m is the same in the four lanes of a query, l its lane's own part of the sum.
struct Running { float m, l; };

// Softmax step over KB blocks of 16 keys: s holds scores and then p (both as four keys a block); returns what the sums so far are multiplied by.
template <int KB>
__device__ __forceinline__ float softmax_step(f32x4 (&s)[KB], Running& r, float scale) {
    float top = kNone;
#pragma unroll
    for (int b = 0; b < KB; ++b) top = fmaxf(fmaxf(fmaxf(top, s[b][0]), fmaxf(s[b][1], s[b][2])), s[b][3]);
    top = over_quarters(top, [](float a, float b) { return fmaxf(a, b); });
    const float m = fmaxf(r.m, top * scale);
    const float base = m == kNone ? 0.f : m;               // nothing seen yet: every p is 0
    const float back = __builtin_amdgcn_exp2f(r.m - base);
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[b][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], scale, -base));
            sum += s[b][e];
        }
    r.m = m;
    r.l = r.l * back + sum;
    return back;
}

// Hides from query `pos` what it may not see of the keys key0 + 16 b + 4 q + e.
template <int KB>
__device__ __forceinline__ void hide(f32x4 (&s)[KB], int key0, int pos, int window) {
    const int q4 = (threadIdx.x & 63) >> 4 << 2;
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int key = key0 + 16 * b + q4 + e;
            if (key > pos || (window && key <= pos - window)) s[b][e] = kNone;
        }
}

__device__ __forceinline__ bf16x8 p_frag(f32x4 a, f32x4 b) {
    return __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]), pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])});
}

// Position of the token of row `row` (of the tile's sequence and head).
__device__ __forceinline__ int pos_of(const AttnArgs& p, const AttnTile& t, int row) { return t.kv - t.n + row / p.group; }
__device__ __forceinline__ const lora_bf16* q_row(const AttnArgs& p, const AttnTile& t, int row) {
    const int tok = row / p.group;
    return p.q + (int64_t)(t.first + tok) * p.ldq + (int64_t)(t.g * p.group + row - tok * p.group) * p.c.D;
}

// Four entries from `d` on of a finished row: o = sum of p v, l = sum of p, m = their reference.
__device__ __forceinline__ void put(const AttnArgs& p, const AttnTile& t, int row, int d, f32x4 o, float m, float l) {
    const int tok = row / p.group, head = t.g * p.group + row - tok * p.group;
    if (p.splits > 1) {
        const int64_t at = (int64_t)t.split * p.T * p.H + (int64_t)(t.first + tok) * p.H + head;
        *(f32x4*)(p.part_o + at * p.c.D + d) = o;
        if (d == 0) {
            p.part_ml[2 * at] = m;
            p.part_ml[2 * at + 1] = l;
        }
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;             // a row that sees nothing: zeros
    u32x2 v;
    v.x = pack_bf16x2(o[0] * inv, o[1] * inv);
    v.y = pack_bf16x2(o[2] * inv, o[3] * inv);
    *(u32x2*)(p.out + (int64_t)(t.first + tok) * p.ldo + (int64_t)head * p.c.D + d) = v;
}

// ---- few rows --------------------------------------------------------------------------------------
// NQ blocks of 16 rows; a wave takes every fourth tile of 32 keys.
template <int D, bool FP8, int NQ>
struct Few {
    static constexpr int KEYS = 32, WAVES = 4;
    static constexpr int KL = 2 * D / (FP8 ? 64 : 32);             // 16-byte loads of a lane for the keys of a tile
    static constexpr int VL = KEYS * D * (FP8 ? 1 : 2) / 1024;     // ... for the values
    static constexpr int V_BYTES = KEYS * D * 2, O_BYTES = 16 * NQ * D * 4;
    static constexpr int WAVE_LDS = V_BYTES > O_BYTES ? V_BYTES : O_BYTES;
    static constexpr int LDS = WAVES * WAVE_LDS + WAVES * NQ * 16 * 8;
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
    f32x4 o[NQ][DB];
    Running run[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        run[i] = Running{kNone, 0.f};
#pragma unroll
        for (int d = 0; d < DB; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    u32x4 kr[C::KL], vr[C::VL];
    uint8_t ke[2], ve[C::VL];
    const char *kc = (const char*)p.c.k, *vc = (const char*)p.c.v;
    constexpr int ESZ = FP8 ? 1 : 2, LANES = D * ESZ / 16;          // lanes to a row of values
    int64_t blk[2];
    auto find = [&](int key) {
#pragma unroll
        for (int b = 0; b < 2; ++b) blk[b] = attn_block(p, t, min(key + 16 * b, t.k1 - 1) & ~15);
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

    int key = t.k0 + C::KEYS * w;
    if (key < t.k1) {
        find(key);
        load_k();
        load_v();
    }
    for (; key < t.k1; key += C::WAVES * C::KEYS) {
        const bool more = key + C::WAVES * C::KEYS < t.k1;
        // values to LDS; a row past the end holds anything, and 0 x anything need not be 0
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < C::VL; ++i) {
            const int row = i * (64 / LANES) + l / LANES, ch = l % LANES;
            const bool in = key + row < t.k1;
            if constexpr (FP8) {
                const float sc = scale_of(ve[i]);
                const bf16x8 lo = widen8(vr[i][0], vr[i][1], sc), hi = widen8(vr[i][2], vr[i][3], sc);
                *(u32x4*)(mine + v_off<D>(row, 2 * ch)) = in ? __builtin_bit_cast(u32x4, lo) : u32x4{0u, 0u, 0u, 0u};
                *(u32x4*)(mine + v_off<D>(row, 2 * ch + 1)) = in ? __builtin_bit_cast(u32x4, hi) : u32x4{0u, 0u, 0u, 0u};
            } else {
                *(u32x4*)(mine + v_off<D>(row, ch)) = in ? vr[i] : u32x4{0u, 0u, 0u, 0u};
            }
        }
        if (more) {
            find(key + C::WAVES * C::KEYS);
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
        const bool whole = key + C::KEYS - 1 <= pos_lo && (!p.window || key > pos_of(p, t, t.row0 + t.rows - 1) - p.window);
        bf16x8 pf[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (!whole) hide(s[i], key, pos[i], p.window);
            const float back = softmax_step(s[i], run[i], p.scale);
            pf[i] = p_frag(s[i][0], s[i][1]);
            if (__any(back != 1.f))
#pragma unroll
                for (int d = 0; d < DB; ++d) o[i][d] *= back;
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            const bf16x8 vf = v_frag<D>(mine, 0, d);
#pragma unroll
            for (int i = 0; i < NQ; ++i) o[i][d] = LF_MFMA(vf, pf[i], o[i][d]);
        }
    }

    // the four waves' sums, brought to one reference
    float* ml = (float*)(smem + C::WAVES * C::WAVE_LDS);              // [row][wave] of m, then of l
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        run[i].l = over_quarters(run[i].l, [](float a, float b) { return a + b; });
        if (q == 0) {
            ml[(16 * i + c) * C::WAVES + w] = run[i].m;
            ml[(NQ * 16 + 16 * i + c) * C::WAVES + w] = run[i].l;
        }
    }
    __syncthreads();
    const auto joined = [&](int row, float& m, float& sum) {
        const f32x4 a = *(const f32x4*)(ml + row * C::WAVES), b = *(const f32x4*)(ml + (NQ * 16 + row) * C::WAVES);
        m = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
        const float base = m == kNone ? 0.f : m;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += b[i] * __builtin_amdgcn_exp2f(a[i] - base);
    };
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        float m, sum;
        joined(16 * i + c, m, sum);
        const float f = __builtin_amdgcn_exp2f(run[i].m - (m == kNone ? 0.f : m));
#pragma unroll
        for (int d = 0; d < DB; ++d) *(f32x4*)(mine + ((16 * i + c) * D + (((4 * d + q) ^ c) << 2)) * 4) = o[i][d] * f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.rows * (D / 4); i += 256) {
        const int row = i / (D / 4), ch = i % (D / 4);
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < C::WAVES; ++k) v += *(const f32x4*)(smem + k * C::WAVE_LDS + (row * D + ((ch ^ (row & 15)) << 2)) * 4);
        float m, sum;
        joined(row, m, sum);
        put(p, t, t.row0 + row, 4 * ch, v, m, sum);
    }
}

// ---- many rows --------------------------------------------------------------------------------------
template <int D>
struct Many {
    static constexpr int KEYS = 64, ROWS = 128, NQ = 2;
    static constexpr int TILE = KEYS * D * 2, STAGE = 2 * TILE, LDS = 2 * STAGE;
};

template <int D, bool FP8>
__global__ void __launch_bounds__(256, 2) attn_many_kernel(AttnArgs p) {
    using C = Many<D>;
    constexpr int NQ = C::NQ, KK = D / 32, DB = D / 16, KB = C::KEYS / 16;
    constexpr int ESZ = FP8 ? 1 : 2, LANES = D * ESZ / 16, RPP = 256 / LANES, L = C::KEYS / RPP;   // rows a pass of the workgroup, passes
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
    const int pos_lo = pos_of(p, t, t.row0 + min(32 * w, t.rows - 1)), pos_hi = pos_of(p, t, t.row0 + min(32 * w + 31, t.rows - 1));
    f32x4 o[NQ][DB];
    Running run[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        run[i] = Running{kNone, 0.f};
#pragma unroll
        for (int d = 0; d < DB; ++d) o[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // a thread brings 16 bytes of a row of keys and one of values in each pass
    u32x4 kr[L], vr[L];
    uint8_t ke[L], ve[L];
    const int row_in = threadIdx.x / LANES, ch = threadIdx.x % LANES;
    auto load = [&](int key) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int row = i * RPP + row_in;
            const int64_t at = attn_block(p, t, min(key + (row & ~15), t.k1 - 1) & ~15) + (row & 15);
            kr[i] = *(const u32x4*)((const char*)p.c.k + at * (D * ESZ) + ch * 16);
            vr[i] = *(const u32x4*)((const char*)p.c.v + at * (D * ESZ) + ch * 16);
            if constexpr (FP8) {
                ke[i] = p.c.k_exp[at];
                ve[i] = p.c.v_exp[at];
            }
        }
    };
    auto store = [&](int key, char* st) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const int row = i * RPP + row_in;
            const u32x4 zero{0u, 0u, 0u, 0u};
            const bool in = key + row < t.k1;              // a row past the end holds anything, and 0 x anything need not be 0
            if constexpr (FP8) {
                const float sk = scale_of(ke[i]), sv = scale_of(ve[i]);
                *(u32x4*)(st + k_off<D>(row, 2 * ch)) = __builtin_bit_cast(u32x4, widen8(kr[i][0], kr[i][1], sk));
                *(u32x4*)(st + k_off<D>(row, 2 * ch + 1)) = __builtin_bit_cast(u32x4, widen8(kr[i][2], kr[i][3], sk));
                const u32x4 lo = __builtin_bit_cast(u32x4, widen8(vr[i][0], vr[i][1], sv)), hi = __builtin_bit_cast(u32x4, widen8(vr[i][2], vr[i][3], sv));
                *(u32x4*)(st + C::TILE + v_off<D>(row, 2 * ch)) = in ? lo : zero;
                *(u32x4*)(st + C::TILE + v_off<D>(row, 2 * ch + 1)) = in ? hi : zero;
            } else {
                *(u32x4*)(st + k_off<D>(row, ch)) = kr[i];
                *(u32x4*)(st + C::TILE + v_off<D>(row, ch)) = in ? vr[i] : zero;
            }
        }
    };

    int stage = 0;
    if (t.k0 < t.k1) {
        load(t.k0);
        store(t.k0, smem);
    }
    __syncthreads();
    for (int key = t.k0; key < t.k1; key += C::KEYS) {
        const bool more = key + C::KEYS < t.k1;
        if (more) load(key + C::KEYS);
        const char* st = smem + stage * C::STAGE;
        // (a wave whose rows see nothing of the tile leaves it out)
        if (key <= pos_hi && (!p.window || key + C::KEYS - 1 > pos_lo - p.window)) {
            f32x4 s[NQ][KB];
#pragma unroll
            for (int b = 0; b < KB; ++b) {
#pragma unroll
                for (int i = 0; i < NQ; ++i) s[i][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < KK; ++kk) {
                    const bf16x8 kf = __builtin_bit_cast(bf16x8, *(const u32x4*)(st + k_off<D>(16 * b + c, 4 * kk + q)));
#pragma unroll
                    for (int i = 0; i < NQ; ++i) s[i][b] = LF_MFMA(kf, qf[i][kk], s[i][b]);
                }
            }
            const bool whole = key + C::KEYS - 1 <= pos_lo && (!p.window || key > pos_hi - p.window);
            bf16x8 pf[NQ][KB / 2];
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                if (!whole) hide(s[i], key, pos[i], p.window);
                const float back = softmax_step(s[i], run[i], p.scale);
#pragma unroll
                for (int b = 0; b < KB / 2; ++b) pf[i][b] = p_frag(s[i][2 * b], s[i][2 * b + 1]);
                if (__any(back != 1.f))
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[i][d] *= back;
            }
#pragma unroll
            for (int b = 0; b < KB / 2; ++b)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const bf16x8 vf = v_frag<D>(st + C::TILE, 32 * b, d);
#pragma unroll
                    for (int i = 0; i < NQ; ++i) o[i][d] = LF_MFMA(vf, pf[i][b], o[i][d]);
                }
        }
        // the other stage was last read before the barrier that began this step
        stage ^= 1;
        if (more) store(key + C::KEYS, smem + stage * C::STAGE);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const float sum = over_quarters(run[i].l, [](float a, float b) { return a + b; });
        const int row = 32 * w + 16 * i + c;
        if (row < t.rows)
#pragma unroll
            for (int d = 0; d < DB; ++d) put(p, t, t.row0 + row, 16 * d + 4 * q, o[i][d], run[i].m, sum);
    }
}

// ---- the parts' results, joined ---------------------------------------------------------------------
// A wave for a row, D / 64 entries to a lane.
template <int D, int BM>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs p) {
    const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    AttnTile t;
    const int per = (p.tiles * BM + 3) / 4;                 // workgroups for a head of a sequence
    int id = blockIdx.x;
    const int row = id % per * 4 + w;
    id /= per;
    t.g = id % p.c.heads;
    t.b = id / p.c.heads;
    t.tile = row / BM;
    if (!attn_rows<BM>(p, t) || row - t.row0 >= t.rows) return;
    const int tok = row / p.group, head = t.g * p.group + row - tok * p.group;
    const int64_t at = (int64_t)(t.first + tok) * p.H + head, plane = (int64_t)p.T * p.H;
    float m = kNone;
    for (int i = 0; i < t.parts; ++i) m = fmaxf(m, p.part_ml[2 * (i * plane + at)]);
    const float base = m == kNone ? 0.f : m;
    constexpr int E = D / 64;
    float sum = 0.f, o[E] = {};
    for (int i = 0; i < t.parts; ++i) {
        const float f = __builtin_amdgcn_exp2f(p.part_ml[2 * (i * plane + at)] - base);
        sum += f * p.part_ml[2 * (i * plane + at) + 1];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += f * p.part_o[(i * plane + at) * D + E * l + e];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    lora_bf16* out = p.out + (int64_t)(t.first + tok) * p.ldo + (int64_t)head * D + E * l;
    if constexpr (E == 1) out[0] = (lora_bf16)(pack_bf16x2(o[0] * inv, 0.f) & 0xFFFFu);
    else *(uint32_t*)out = pack_bf16x2(o[0] * inv, o[1] * inv);
}

// ---- launches ---------------------------------------------------------------------------------------
AttnPlan plan_attn(int B, int G, int group, int D, int max_new, int64_t max_kv, int window) {
    AttnPlan pl;
    const int64_t rows = (int64_t)max_new * group;
    pl.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 128;
    const int64_t tiles = (rows + pl.rows - 1) / pl.rows;
    // the most keys that a tile sees
    int64_t keys = max_kv;
    if (window) keys = std::min<int64_t>(keys, (int64_t)window + (pl.rows + group - 1) / group + 16);
    // parts of 256 keys and more, until there are four (few rows) or two workgroups to a compute unit
    const int64_t want = (pl.rows == 128 ? 2 : 4) * kComputeUnits, have = tiles * B * G;
    int64_t parts = std::max<int64_t>(1, std::min(want / std::max<int64_t>(have, 1), (keys + 255) / 256));
    const int64_t step = 128;
    pl.split_keys = (int)(((keys + parts - 1) / parts + step - 1) / step * step);
    if (pl.split_keys < step) pl.split_keys = step;
    pl.splits = (int)std::max<int64_t>(1, (keys + pl.split_keys - 1) / pl.split_keys);
    if (pl.splits == 1) pl.split_keys = 1 << 30;
    return pl;
}

template <class K>
static hipError_t launch_lds(K kernel, int lds, unsigned blocks, const AttnArgs& a, hipStream_t st) {
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), lds, st, a);
    return hipGetLastError();
}

template <int D, bool FP8>
static hipError_t launch_attn_t(const AttnArgs& a, int rows, unsigned blocks, hipStream_t st) {
    if (rows == 16) return launch_lds(attn_few_kernel<D, FP8, 1>, Few<D, FP8, 1>::LDS, blocks, a, st);
    if (rows == 32) return launch_lds(attn_few_kernel<D, FP8, 2>, Few<D, FP8, 2>::LDS, blocks, a, st);
    return launch_lds(attn_many_kernel<D, FP8>, Many<D>::LDS, blocks, a, st);
}

template <int D>
static hipError_t launch_join(const AttnArgs& a, int rows, hipStream_t st) {
    const int64_t blocks = (int64_t)((a.tiles * (int64_t)rows + 3) / 4) * a.c.heads * a.B;
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
    return a.c.D == 64 ? launch_join<64>(a, p.rows, st) : launch_join<128>(a, p.rows, st);
}

}  // namespace lf
