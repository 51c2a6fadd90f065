// Arguments of the operators around served adapters (lf_rope.hip, lf_cache.hip, lf_attn.hip, lf_requests.hip; entry points and checks in
// lf_serve_api.hip), and device pieces that they share.
#pragma once
#include "lf_internal.h"
#include "lf_quant.h"

namespace lf {

// Norm of queries and keys and their rotation; the heads of a row lie side by side, rows ld* elements apart.
struct RopeArgs {
    const lora_bf16* q; const lora_bf16* k;
    const lora_bf16* gamma_q; const lora_bf16* gamma_k;
    const float* cos_; const float* sin_;       // [positions, rot / 2]
    const int32_t* pos;
    lora_bf16* q_out; lora_bf16* k_out;         // backward: dq, dk
    const lora_bf16* dq_out; const lora_bf16* dk_out;
    float* part;                                // backward: [blocks, 2, D] partial sums of dgamma
    int64_t ldq, ldk, ldqo, ldko, lddq, lddk;   // dq_out, dk_out: lddq, lddk
    int64_t M;
    int H, G, D, rot, positions, parts;
    float eps;
};
struct RopeFinalizeArgs { const float* part; float* dgamma_q; float* dgamma_k; int blocks, D, accumulate; };

// Paged cache: k, v [pages, heads, page, D], fp8 also k_exp, v_exp [pages, heads, page], 4 bits [.., page, D / 32].
constexpr int kCacheBf16 = 0, kCacheFp8 = 1, kCacheFp4 = 2;
struct PagedCache {
    void* k; void* v; uint8_t* k_exp; uint8_t* v_exp;
    int64_t pages;
    int page_shift, heads, D, form;
};
struct CacheCopyArgs {
    PagedCache c;
    lora_bf16* k; lora_bf16* v;                 // write: inputs; read: outputs
    const int64_t* slots;
    int64_t ldk, ldv, M;
};

// Norm (if gamma_q and gamma_k are given) and rotation of queries and keys; queries out, keys and values into slots of a cache of G = c.heads heads.
struct AppendArgs {
    PagedCache c;
    const lora_bf16* q; const lora_bf16* k; const lora_bf16* v;
    const lora_bf16* gamma_q; const lora_bf16* gamma_k;
    const float* cos_; const float* sin_;       // [positions, rot / 2]
    const int32_t* pos; const int64_t* slots;
    lora_bf16* q_out;
    int64_t ldq, ldk, ldv, ldqo, M;
    int H, rot, positions, parts, kv_parts, kv_blocks;
    float eps;
};

// Weights in 4 bits: codes [N, K / 2], exps [N, K / 32]; W [N, K].
struct WeightsArgs { lora_bf16* W; uint8_t* codes; uint8_t* exps; int64_t entries; };

struct AttnArgs {
    PagedCache c;
    const lora_bf16* q; lora_bf16* out;
    const int32_t* table; const int32_t* offsets; const int32_t* kv_lens;
    float* part_o; float* part_ml;              // splits > 1: [splits, T * H, D], [splits, T * H, 2]
    int64_t ldq, ldo, ldt;
    int T, B, H, group;                         // group: query heads of a key/value head
    int max_pages, window;                      // pages of a table row; 0: no window
    int tiles, splits, split_keys;              // row tiles of the longest chunk; parts of a key range and their length
    float scale;                                // of the scores, times log2 e
};
struct AttnPlan { int rows, splits, split_keys; };      // query rows (token, head of the group) of a workgroup

// The layer of many requests; W, or its codes and exponents.
struct RequestArgs {
    const lora_bf16* X; const lora_bf16* W; const lora_bf16* A; const lora_bf16* B;
    const int32_t* ids; const int32_t* ranks; const float* s;
    lora_bf16* Y; lora_bf16* S;
    int M, K, N, r, P;
};
struct QuantisedRequestArgs { RequestArgs r; const uint8_t* codes; const uint8_t* exps; };     // r.P == 0: no adapters
struct QuantisedTiles { int rows, columns, ring_blocks; bool own_term; };

int rope_blocks(int64_t M, int H, int G, int D);        // of the backward: planes of partial sums
hipError_t launch_rope_fwd(RopeArgs a, bool interleaved, hipStream_t st);
hipError_t launch_rope_bwd(RopeArgs a, bool interleaved, const RopeFinalizeArgs& f, hipStream_t st);
hipError_t launch_append(AppendArgs a, bool interleaved, hipStream_t st);
hipError_t launch_weights_write(const WeightsArgs& a, hipStream_t st);
hipError_t launch_weights_read(const WeightsArgs& a, hipStream_t st);
hipError_t launch_cache_write(const CacheCopyArgs& a, hipStream_t st);
hipError_t launch_cache_read(const CacheCopyArgs& a, hipStream_t st);
AttnPlan plan_attn(int B, int G, int group, int D, int max_new, int64_t max_kv, int window, int form);
int64_t attn_part_rows(int64_t T, int B, int G, int group, int max_new, int64_t max_kv, int window, int form);      // of any step of at most these sizes
hipError_t launch_attn(AttnArgs a, const AttnPlan& p, int max_new, hipStream_t st);
hipError_t launch_request_down(const RequestArgs& a, hipStream_t st);       // S alone
hipError_t launch_requests(const RequestArgs& a, hipStream_t st);
QuantisedTiles quantised_tiles(int M, int K, int N, int r, int P);
hipError_t launch_quantised_requests(const QuantisedRequestArgs& a, hipStream_t st);

// ---- device pieces ------------------------------------------------------------------------------
__device__ __forceinline__ void unpack8(u32x4 v, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
    return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}

// Head of a slot, in heads (rows of D entries) from the cache's start.
__device__ __forceinline__ int64_t head_of_slot(const PagedCache& c, int64_t slot, int head) {
    const int64_t page = slot >> c.page_shift;
    return ((page * c.heads + head) << c.page_shift) + (slot - (page << c.page_shift));
}

// Lane j's eight entries of a head that lies in GL lanes, into the cache's head `at`, in its form.  held: they go there (all lanes of a head take part).
template <int GL>
__device__ __forceinline__ void hold_quantised(const PagedCache& c, bool keys, bool held, int64_t at, int j, const float (&x)[8]) {
    uint32_t e;
    if (c.form == kCacheFp8) {
        const u32x2 code = to_fp8<GL>(x, e);
        if (!held) return;
        *(u32x2*)((uint8_t*)(keys ? c.k : c.v) + at * c.D + 8 * j) = code;
        if (j == 0) (keys ? c.k_exp : c.v_exp)[at] = (uint8_t)e;
    } else {
        const uint32_t code = to_fp4(x, e);
        if (!held) return;
        *(uint32_t*)((uint8_t*)(keys ? c.k : c.v) + at * (c.D / 2) + 4 * j) = code;
        if (j % 4 == 0) (keys ? c.k_exp : c.v_exp)[at * (c.D / 32) + j / 4] = (uint8_t)e;
    }
}
template <int GL>
__device__ __forceinline__ void hold_head(const PagedCache& c, bool keys, bool held, int64_t at, int j, u32x4 raw) {
    if (c.form == kCacheBf16) {
        if (held) *(u32x4*)((lora_bf16*)(keys ? c.k : c.v) + at * c.D + 8 * j) = raw;
        return;
    }
    float x[8];
    unpack8(raw, x);
    hold_quantised<GL>(c, keys, held, at, j, x);
}

// Maximum (sum) over the four lanes of a wave that share l & 15.
template <class F>
__device__ __forceinline__ float over_quarters(float x, F&& f) {
    auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    const float y = f(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, y), __builtin_bit_cast(uint32_t, y), false, false);
    return f(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

}  // namespace lf
