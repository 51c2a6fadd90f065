// Device pieces of the norm of queries and keys with their rotation (lf_rope.hip, lf_append.hip).
#pragma once
#include "lf_serve.h"

namespace lf {

// GL lanes to a head, a wave for a row, or for a part of its heads.
template <int GL, bool INTER>
struct RopeLane {
    int j, slot;                       // lane of the head, head of the wave
    bool active, turned;               // ... has entries; they are in the rotated part
    int at, other;                     // first index into a row of the tables; wave lane with the other entries of this one's pairs
    float sign;                        // of the sine in y: - for the first entry of a pair
    uint32_t even, odd;                // bytes of a word of two entries that hold the other entry of the even and of the odd one's pair (v_perm_b32: 0x0c is a zero)
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
        even = !turned ? 0x0c0c0c0cu : INTER ? 0x03020c0cu : 0x01000c0cu;
        odd = !turned ? 0x0c0c0c0cu : INTER ? 0x01000c0cu : 0x03020c0cu;
    }
};

template <int GL>
__device__ __forceinline__ float sum_over_head(float v) {
#pragma unroll
    for (int o = GL / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// Cosine and (signed) sine of each of a lane's entries.  Entries that are not turned: 1 and -0, which times the 0 that others() gives them adds nothing, not even to a -0.
template <int GL, bool INTER, class Args>
__device__ __forceinline__ void angles(const Args& p, const RopeLane<GL, INTER>& ln, int pos, bool known, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = -0.f; }
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

// The other entries of this lane's pairs; zeros where nothing is turned (0 times an infinity that stands there would be NaN): by the lane's selectors at no instruction more, or,
// SELECTED, where there is no register for those, by a select for two entries.
template <bool SELECTED = false, int GL, bool INTER>
__device__ __forceinline__ void others(const RopeLane<GL, INTER>& ln, u32x4 raw, float (&o)[8]) {
    if constexpr (!INTER)
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = (uint32_t)__shfl((int)raw[i], ln.other);
    if constexpr (SELECTED) {
        static_assert(!INTER, "the entries of a word change places by the selectors");
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = ln.turned ? raw[i] : 0u;
        unpack8(raw, o);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[2 * i] = __builtin_bit_cast(float, __builtin_amdgcn_perm(raw[i], raw[i], ln.even));
            o[2 * i + 1] = __builtin_bit_cast(float, __builtin_amdgcn_perm(raw[i], raw[i], ln.odd));
        }
    }
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

template <class F>
inline auto with_lanes(int D, F&& f) {
    if (D <= 64) return f(std::integral_constant<int, 8>{});
    if (D <= 128) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, 32>{});
}

template <class F>
inline hipError_t with_pairs(bool interleaved, F&& f) { return interleaved ? f(std::true_type{}) : f(std::false_type{}); }

}  // namespace lf
