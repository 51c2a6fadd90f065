// Weights into 4 bits (e2m1 and a power of two for 32 entries of a row, lf_quant.h) and back to bf16, which holds their values exactly.  Bound by HBM: 2 + 17 / 32
// bytes an entry.  Rows are whole groups, so that a matrix is one run of entries; eight to a lane, four times.  Measured: 1024 x 4096 written 4.1 us, read 3.8 (11 MB: launch and
// one latency); 14336 x 4096 read 27.1 us (149 MB, 5.5 TB/s).
#include <algorithm>

#include "lf_serve.h"

namespace lf {

constexpr int kWeightsUnroll = 4;                // eight entries each of a lane, under way together

template <bool WRITE>
__global__ void __launch_bounds__(256) weights_kernel(WeightsArgs p) {
    constexpr int U = kWeightsUnroll;
    const int64_t eights = p.entries / 8, first = (int64_t)blockIdx.x * (256 * U) + threadIdx.x;
    if constexpr (WRITE) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = u32x4{0u, 0u, 0u, 0u};
            if (first + 256 * u < eights) raw[u] = *(const u32x4*)(p.W + 8 * (first + 256 * u));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = first + 256 * u;
            float x[8];
            unpack8(raw[u], x);
            uint32_t e;
            const uint32_t code = to_fp4(x, e);
            if (i >= eights) continue;
            *(uint32_t*)(p.codes + 4 * i) = code;
            if (i % 4 == 0) p.exps[i / 4] = (uint8_t)e;
        }
    } else {
        uint32_t code[U], e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = std::min(first + 256 * u, eights - 1);
            code[u] = *(const uint32_t*)(p.codes + 4 * i);
            e[u] = p.exps[i / 4];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + 256 * u < eights) *(u32x4*)(p.W + 8 * (first + 256 * u)) = __builtin_bit_cast(u32x4, from_fp4(code[u], exp2_of_biased(e[u])));
    }
}

template <bool WRITE>
static hipError_t launch_weights(WeightsArgs a, hipStream_t st) {
    // (a launch has fewer than 2^32 threads)
    constexpr int64_t MOST = 1ll << 34;
    hipError_t e = hipSuccess;
    for (int64_t left = a.entries; left > 0 && e == hipSuccess; left -= MOST) {
        a.entries = std::min(left, MOST);
        const int64_t blocks = (a.entries / 8 + 256 * kWeightsUnroll - 1) / (256 * kWeightsUnroll);
        hipLaunchKernelGGL(weights_kernel<WRITE>, dim3((unsigned)blocks), dim3(256), 0, st, a);
        e = hipGetLastError();
        a.W += a.entries;
        a.codes += a.entries / 2;
        a.exps += a.entries / 32;
    }
    return e;
}

hipError_t launch_weights_write(const WeightsArgs& a, hipStream_t st) { return launch_weights<true>(a, st); }
hipError_t launch_weights_read(const WeightsArgs& a, hipStream_t st) { return launch_weights<false>(a, st); }

}  // namespace lf
