// Keys and values into the slots of a paged cache, and back.  In the fp8 form a token's head is held as e4m3 values and one power of two,
// the smallest that keeps its largest magnitude within 448: a scale that costs no rounding of its own, so that a value is rounded once, to
// three fraction bits, and what is read back (value x scale) is exact in bf16.  Bound by HBM: 3 + 1 / D bytes an element (bf16: 4).  Eight
// entries to a lane, a head to 8, 16 or 32 lanes, whose largest magnitude comes from the bit patterns (integers in the order of the values).
// Measured: 2085 tokens of 8 heads of 128 to fp8, 13 MB, 5.5 us (slot, then the head: two latencies), 32768 tokens, 203 MB, 56 us; 29999 tokens read back from
// fp8, 185 MB, 44 us; with two or four heads to a lane, all their loads under way, 48.
#include "lf_serve.h"

namespace lf {

constexpr int kLeastExponent = -117;             // 2^-9 (the least e4m3) times that is still a normal bf16

__device__ __forceinline__ int64_t head_of_slot(const PagedCache& c, int64_t slot, int head) {
    const int64_t page = slot >> c.page_shift;
    return ((page * c.heads + head) << c.page_shift) + (slot - (page << c.page_shift));
}

template <int GL>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheCopyArgs p) {
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / GL;       // token, head
    const int j = threadIdx.x % GL;
    const bool keys = blockIdx.y == 0;
    const int64_t t = item / p.c.heads;
    if (t >= p.M) return;
    const int head = (int)(item - t * p.c.heads);
    const int64_t slot = p.slots[t];
    const bool held = slot >= 0 && slot < p.c.pages << p.c.page_shift && 8 * j < p.c.D;
    u32x4 raw = u32x4{0u, 0u, 0u, 0u};
    if (held) raw = *(const u32x4*)((keys ? p.k + t * p.ldk : p.v + t * p.ldv) + (int64_t)head * p.c.D + 8 * j);
    const int64_t at = held ? head_of_slot(p.c, slot, head) : 0;
    if (!p.c.fp8) {
        if (held) *(u32x4*)((lora_bf16*)(keys ? p.c.k : p.c.v) + at * p.c.D + 8 * j) = raw;
        return;
    }
    // largest finite magnitude; what is not finite becomes the format's NaN
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = raw[i] & 0x7FFFu, hi = raw[i] >> 16 & 0x7FFFu;
        top = max(top, max(lo < 0x7F80u ? lo : 0u, hi < 0x7F80u ? hi : 0u));
    }
#pragma unroll
    for (int o = GL / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const int e = top ? max((int)(top >> 7) - 135 + ((top & 0x7Fu) > 0x60u), kLeastExponent) : 0;     // 448 = 1.75 x 2^8
    const float scale = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    float x[8];
    unpack8(raw, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (__builtin_bit_cast(uint32_t, x[i]) & 0x7F800000u) == 0x7F800000u ? __builtin_nanf("") : x[i] * scale;
    u32x2 code;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
        code[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], v, true);
    }
    if (!held) return;
    *(u32x2*)((uint8_t*)(keys ? p.c.k : p.c.v) + at * p.c.D + 8 * j) = code;
    if (j == 0) (keys ? p.c.k_exp : p.c.v_exp)[at] = (uint8_t)(e + 127);
}

template <int GL, bool PAST>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheCopyArgs p) {
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / GL;
    const int j = threadIdx.x % GL;
    const bool keys = blockIdx.y == 0;
    const int64_t t = item / p.c.heads;
    if (t >= p.M || 8 * j >= p.c.D) return;
    const int head = (int)(item - t * p.c.heads);
    const int64_t slot = p.slots[t];
    u32x4 out = u32x4{0u, 0u, 0u, 0u};
    if (slot >= 0 && slot < p.c.pages << p.c.page_shift) {
        const int64_t at = head_of_slot(p.c, slot, head);
        if (p.c.fp8) {
            const u32x2 code = *(const u32x2*)((const uint8_t*)(keys ? p.c.k : p.c.v) + at * p.c.D + 8 * j);
            const int e = (int)(keys ? p.c.k_exp : p.c.v_exp)[at] - 127;
            float x[8];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)code[i], true);
                x[4 * i] = ldexpf(lo[0], e);
                x[4 * i + 1] = ldexpf(lo[1], e);
                x[4 * i + 2] = ldexpf(hi[0], e);
                x[4 * i + 3] = ldexpf(hi[1], e);
            }
            out = pack8(x);
        } else {
            out = *(const u32x4*)((const lora_bf16*)(keys ? p.c.k : p.c.v) + at * p.c.D + 8 * j);
        }
    }
    u32x4* to = (u32x4*)((keys ? p.k + t * p.ldk : p.v + t * p.ldv) + (int64_t)head * p.c.D + 8 * j);
    if constexpr (PAST) __builtin_nontemporal_store(out, to);
    else *to = out;
}

template <class F>
static hipError_t with_lanes(const CacheCopyArgs& a, F&& f) {
    if (a.c.D <= 64) return f(std::integral_constant<int, 8>{});
    if (a.c.D <= 128) return f(std::integral_constant<int, 16>{});
    return f(std::integral_constant<int, 32>{});
}

hipError_t launch_cache_write(const CacheCopyArgs& a, hipStream_t st) {
    return with_lanes(a, [&](auto gl) {
        const int64_t blocks = (a.M * a.c.heads * gl() + 255) / 256;
        hipLaunchKernelGGL(cache_write_kernel<gl()>, dim3((unsigned)blocks, 2), dim3(256), 0, st, a);
        return hipGetLastError();
    });
}

// Outputs of 176 MB and more, which the 256 MB memory-side cache does not hold beside what is read, go past the caches.  us, stored / past the caches, alone
// and with the reading of the outputs by another kernel behind, three sets in turn, fp8, 8 heads of 128: 16000 tokens (66 MB) 25.7 / 18.4, 48.3 / 51.7; 29999
// (123 MB) 44.6 / 30.6, 85 / 89; 36000 53.4 / 36.6, 104.5 / 105.3; 48000 (197 MB) 69.6 / 65.8, 139.5 / 135.8; 72000 104.1 / 96.4, 206.2 / 199.6; bf16, 16000
// 26.2 / 21.0, 48.6 / 53.5; from 48000 on level with the reader.
hipError_t launch_cache_read(const CacheCopyArgs& a, hipStream_t st) {
    return with_lanes(a, [&](auto gl) {
        const int64_t blocks = (a.M * a.c.heads * gl() + 255) / 256;
        if (a.M * a.c.heads * a.c.D * 4 >= 176 << 20) hipLaunchKernelGGL((cache_read_kernel<gl(), true>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((cache_read_kernel<gl(), false>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a);
        return hipGetLastError();
    });
}

}  // namespace lf
