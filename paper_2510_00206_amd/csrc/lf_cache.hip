// Keys and values into the slots of a paged cache, and back.  In the fp8 form a token's head is held as e4m3 values and one power of two, in the 4-bit form as
// e2m1 values and one power of two for 32 entries (lf_quant.h): a value is rounded once, to three fraction bits or one, and what is read back
// (value x scale) is exact in bf16.  Bound by HBM: 3 + 1 / D bytes an element (bf16: 4; 4 bits: 2 + 17 / 32).  Eight entries to a lane, a head to 8, 16
// or 32 lanes.
// Measured in a captured graph, us: tokens of 8 heads of 128 to fp8, 2085 (13 MB) 4.75 (slot, then the head: two latencies), 32768 (203 MB) 50.9, to bf16 4.6 and 53.6; 29999
// tokens read back from fp8, 185 MB, 44; with two or four heads to a lane, all their loads under way, 48.
#include "lf_quant.h"
#include "lf_serve.h"

namespace lf {

// A kernel for each form: 8 waves to a SIMD and some 250 instructions each are most of what 2085 tokens take, so that what is not of the form counts.
template <int GL, int FORM>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheCopyArgs p) {
    p.c.form = FORM;
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
    hold_head<GL>(p.c, keys, held, at, j, raw);
}

// FOUR: 4 bits, in kernels of their own; as a third branch they cost the other forms' reading 1.2 us of 43.7.
template <int GL, bool PAST, bool FOUR>
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
        if constexpr (FOUR) {
            const uint32_t code = *(const uint32_t*)((const uint8_t*)(keys ? p.c.k : p.c.v) + at * (p.c.D / 2) + 4 * j);
            out = __builtin_bit_cast(u32x4, from_fp4(code, exp2_of_biased((keys ? p.c.k_exp : p.c.v_exp)[at * (p.c.D / 32) + j / 4])));
        } else if (p.c.form == kCacheFp8) {
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
        const auto launch = [&](auto form) { hipLaunchKernelGGL((cache_write_kernel<gl(), form()>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a); };
        if (a.c.form == kCacheFp4) launch(std::integral_constant<int, kCacheFp4>{});
        else if (a.c.form == kCacheFp8) launch(std::integral_constant<int, kCacheFp8>{});
        else launch(std::integral_constant<int, kCacheBf16>{});
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
        const auto launch = [&](auto past, auto four) { hipLaunchKernelGGL((cache_read_kernel<gl(), past(), four()>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a); };
        const std::true_type yes;
        const std::false_type no;
        const bool past = a.M * a.c.heads * a.c.D * 4 >= 176 << 20;
        if (a.c.form == kCacheFp4) past ? launch(yes, yes) : launch(no, yes);
        else past ? launch(yes, no) : launch(no, no);
        return hipGetLastError();
    });
}

}  // namespace lf
