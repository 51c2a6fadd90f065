// C ABI of the operators around served adapters: checks of the arguments and launches.  Nothing here allocates device memory or
// synchronises; every kernel goes to the caller's stream.
#include <math.h>

#include <algorithm>

#include "../../include/lorafusion.h"
#include "lf_serve.h"

using namespace lf;

namespace {

inline bool misaligned(const void* p, size_t a = 16) { return ((uintptr_t)p & (a - 1)) != 0; }
inline lora_status done(hipError_t e) { return e == hipSuccess ? LORA_OK : LORA_ERR_HIP; }
inline size_t align_up(size_t v, size_t a = 256) { return (v + a - 1) / a * a; }

// Heads side by side in rows `ld` elements apart.
inline bool bad_stride(int64_t ld, int64_t heads, int64_t dim) { return ld < heads * dim || (ld & 7) || ld >= (1ll << 31); }

lora_status check_heads(int64_t M, int32_t H, int32_t G, int32_t D) {
    if (M < 0 || H < 1 || G < 1 || D < 1) return LORA_ERR_SHAPE;
    if ((D & 15) || D > 256 || H > 1024 || G > 1024 || M >= (1ll << 26)) return LORA_ERR_UNSUPPORTED;
    return LORA_OK;
}

lora_status check_rope(int64_t M, int32_t H, int32_t G, int32_t D, int32_t rot, int64_t positions, float eps) {
    const lora_status st = check_heads(M, H, G, D);
    if (st != LORA_OK) return st;
    if (positions < 0 || positions >= (1ll << 31)) return LORA_ERR_SHAPE;
    if (rot < 16 || rot > D || (rot & 15)) return LORA_ERR_UNSUPPORTED;
    if (!(eps > 0.f) || !isfinite(eps)) return LORA_ERR_PARAM;
    return LORA_OK;
}

lora_status paged(const lora_kv_cache* c, PagedCache& out) {
    if (!c || !c->k || !c->v || (c->fp8 && (!c->k_exp || !c->v_exp))) return LORA_ERR_NULL;
    if (c->pages < 1 || c->heads < 1 || c->dim < 1 || c->page < 1) return LORA_ERR_SHAPE;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)) || c->heads > 1024 || c->pages >= (1ll << 31) || (c->dim & 15) || c->dim > 256)
        return LORA_ERR_UNSUPPORTED;
    if (misaligned(c->k) || misaligned(c->v)) return LORA_ERR_ALIGN;
    out = PagedCache{c->k, c->v, c->k_exp, c->v_exp, c->pages, __builtin_ctz((unsigned)c->page), c->heads, c->dim, c->fp8 != 0};
    return LORA_OK;
}

lora_status cache_copy(const lora_kv_cache* cache, const void* k, const void* v, int64_t ldk, int64_t ldv, const int64_t* slots, int64_t M, CacheCopyArgs& a) {
    const lora_status st = paged(cache, a.c);
    if (st != LORA_OK) return st;
    if (M < 0) return LORA_ERR_SHAPE;
    if (M == 0) return LORA_OK;
    if (!k || !v || !slots) return LORA_ERR_NULL;
    if (bad_stride(ldk, cache->heads, cache->dim) || bad_stride(ldv, cache->heads, cache->dim)) return LORA_ERR_SHAPE;
    if (misaligned(k) || misaligned(v) || misaligned(slots, 8)) return LORA_ERR_ALIGN;
    // (threads of a launch, in whole workgroups of 256; 32 lanes to a head at most)
    if (M > ((1ll << 32) - 256) / (32ll * cache->heads)) return LORA_ERR_UNSUPPORTED;
    a.k = (lora_bf16*)k;
    a.v = (lora_bf16*)v;
    a.slots = slots;
    a.ldk = ldk;
    a.ldv = ldv;
    a.M = M;
    return LORA_OK;
}

lora_status check_attn(const PagedCache& c, int64_t T, int32_t H, int64_t B, int64_t max_new, int64_t max_kv, int32_t window) {
    if (T < 0 || B < 0 || H < 1 || max_new < 0 || max_kv < 0 || window < 0 || H % c.heads) return LORA_ERR_SHAPE;
    const int64_t most = 0x7FFFFFFF / H;                   // (T * H could wrap)
    if (!(c.D == 64 || c.D == 128) || T > most || max_new > most || max_kv >= (1ll << 30) || B >= (1ll << 31) || window >= (1 << 30))
        return LORA_ERR_UNSUPPORTED;
    return LORA_OK;
}

size_t attn_scratch(size_t part_rows, int32_t D) { return align_up(part_rows * D * 4) + align_up(part_rows * 8); }
size_t attn_scratch(const AttnPlan& pl, int64_t T, int32_t H, int32_t D) { return pl.splits == 1 ? 0 : attn_scratch((size_t)pl.splits * T * H, D); }

}  // namespace

extern "C" {

lora_status lora_requests_fwd(const lora_bf16* X, const lora_bf16* W, const lora_bf16* A, const lora_bf16* B, const int32_t* ids,
                              const int32_t* ranks, const float* s, int64_t M, int64_t K, int64_t N, int32_t r, int64_t P, lora_bf16* Y,
                              lora_bf16* S, lora_stream stream) {
    if (M < 0 || K <= 0 || N <= 0 || M >= (1ll << 31) || K >= (1ll << 31) || N >= (1ll << 31) || P < 1 || P >= (1ll << 31)) return LORA_ERR_SHAPE;
    if ((K & 63) || (N & 63) || K > (1 << 22) || N > (1 << 22) || !(r == 16 || r == 32 || r == 64) || M >= (1 << 21)) return LORA_ERR_UNSUPPORTED;
    if (!W || !A || !B || !s || (M > 0 && (!X || !ids || !Y || !S))) return LORA_ERR_NULL;
    if (misaligned(X) || misaligned(W) || misaligned(A) || misaligned(B) || misaligned(Y) || misaligned(S)) return LORA_ERR_ALIGN;
    if (misaligned(ids, 4) || misaligned(ranks, 4) || misaligned(s, 4)) return LORA_ERR_ALIGN;
    if (M == 0) return LORA_OK;
    return done(launch_requests(RequestArgs{X, W, A, B, ids, ranks, s, Y, S, (int)M, (int)K, (int)N, r, (int)P}, (hipStream_t)stream));
}

lora_status lora_qk_norm_rope_fwd(const lora_bf16* q, const lora_bf16* k, const lora_bf16* gamma_q, const lora_bf16* gamma_k,
                                  const float* cos_table, const float* sin_table, const int32_t* pos, int64_t M, int32_t H, int32_t G, int32_t D,
                                  int32_t rot, int64_t positions, int64_t ldq, int64_t ldk, int64_t ldqo, int64_t ldko, float eps,
                                  int interleaved, lora_bf16* q_out, lora_bf16* k_out, lora_stream stream) {
    const lora_status st = check_rope(M, H, G, D, rot, positions, eps);
    if (st != LORA_OK) return st;
    if (!gamma_q || !gamma_k || (positions && (!cos_table || !sin_table)) || (M > 0 && (!q || !k || !pos || !q_out || !k_out))) return LORA_ERR_NULL;
    if (bad_stride(ldq, H, D) || bad_stride(ldqo, H, D) || bad_stride(ldk, G, D) || bad_stride(ldko, G, D)) return LORA_ERR_SHAPE;
    if (misaligned(q) || misaligned(k) || misaligned(gamma_q) || misaligned(gamma_k) || misaligned(cos_table) || misaligned(sin_table) ||
        misaligned(pos, 4) || misaligned(q_out) || misaligned(k_out))
        return LORA_ERR_ALIGN;
    if (M == 0) return LORA_OK;
    RopeArgs a{q, k, gamma_q, gamma_k, cos_table, sin_table, pos, q_out, k_out, nullptr, nullptr, nullptr, ldq, ldk, ldqo, ldko, 0, 0, M, H, G, D, rot,
               (int)positions, 1, eps};
    return done(launch_rope_fwd(a, interleaved != 0, (hipStream_t)stream));
}

size_t lora_qk_norm_rope_workspace_bytes(int64_t M, int32_t H, int32_t G, int32_t D) {
    if (check_heads(M, H, G, D) != LORA_OK) return 0;
    return std::max<size_t>(256, align_up((size_t)rope_blocks(M, H, G, D) * 2 * D * 4));
}

lora_status lora_qk_norm_rope_bwd(const lora_bf16* q, const lora_bf16* k, const lora_bf16* gamma_q, const lora_bf16* gamma_k,
                                  const float* cos_table, const float* sin_table, const int32_t* pos, const lora_bf16* dq_out,
                                  const lora_bf16* dk_out, int64_t M, int32_t H, int32_t G, int32_t D, int32_t rot, int64_t positions, int64_t ldq,
                                  int64_t ldk, int64_t lddqo, int64_t lddko, int64_t lddq, int64_t lddk, float eps, int interleaved, lora_bf16* dq,
                                  lora_bf16* dk, float* dgamma_q, float* dgamma_k, int accumulate, void* workspace, size_t workspace_bytes,
                                  lora_stream stream) {
    const lora_status st = check_rope(M, H, G, D, rot, positions, eps);
    if (st != LORA_OK) return st;
    if (!gamma_q || !gamma_k || !dgamma_q || !dgamma_k || !workspace || (positions && (!cos_table || !sin_table)) ||
        (M > 0 && (!q || !k || !pos || !dq_out || !dk_out || !dq || !dk)))
        return LORA_ERR_NULL;
    if (bad_stride(ldq, H, D) || bad_stride(lddqo, H, D) || bad_stride(lddq, H, D) || bad_stride(ldk, G, D) || bad_stride(lddko, G, D) ||
        bad_stride(lddk, G, D))
        return LORA_ERR_SHAPE;
    if (misaligned(q) || misaligned(k) || misaligned(gamma_q) || misaligned(gamma_k) || misaligned(cos_table) || misaligned(sin_table) ||
        misaligned(pos, 4) || misaligned(dq_out) || misaligned(dk_out) || misaligned(dq) || misaligned(dk) || misaligned(dgamma_q) ||
        misaligned(dgamma_k) || misaligned(workspace, 256))
        return LORA_ERR_ALIGN;
    if (workspace_bytes < lora_qk_norm_rope_workspace_bytes(M, H, G, D)) return LORA_ERR_WORKSPACE;
    RopeArgs a{q, k, gamma_q, gamma_k, cos_table, sin_table, pos, dq, dk, dq_out, dk_out, (float*)workspace, ldq, ldk, lddq, lddk, lddqo, lddko, M, H, G, D,
               rot, (int)positions, 1, eps};
    const RopeFinalizeArgs f{(const float*)workspace, dgamma_q, dgamma_k, rope_blocks(M, H, G, D), D, accumulate != 0};
    return done(launch_rope_bwd(a, interleaved != 0, f, (hipStream_t)stream));
}

lora_status lora_kv_cache_write(const lora_kv_cache* cache, const lora_bf16* k, const lora_bf16* v, int64_t ldk, int64_t ldv, const int64_t* slots,
                                int64_t M, lora_stream stream) {
    CacheCopyArgs a{};
    const lora_status st = cache_copy(cache, k, v, ldk, ldv, slots, M, a);
    return st != LORA_OK || M == 0 ? st : done(launch_cache_write(a, (hipStream_t)stream));
}

lora_status lora_kv_cache_read(const lora_kv_cache* cache, const int64_t* slots, int64_t M, lora_bf16* k, lora_bf16* v, int64_t ldk, int64_t ldv,
                               lora_stream stream) {
    CacheCopyArgs a{};
    const lora_status st = cache_copy(cache, k, v, ldk, ldv, slots, M, a);
    return st != LORA_OK || M == 0 ? st : done(launch_cache_read(a, (hipStream_t)stream));
}

size_t lora_paged_attn_workspace_bytes(const lora_kv_cache* cache, int64_t T, int32_t H, int64_t B, int64_t max_new, int64_t max_kv, int32_t window) {
    PagedCache c;
    if (paged(cache, c) != LORA_OK || check_attn(c, T, H, B, max_new, max_kv, window) != LORA_OK) return 0;
    if (T == 0 || B == 0 || max_new == 0) return 256;
    const int group = H / c.heads;
    // (its own plan too: more tokens than sequences of max_new can have are allowed)
    return std::max({(size_t)256, attn_scratch(plan_attn((int)B, c.heads, group, c.D, (int)max_new, max_kv, window), T, H, c.D),
                     attn_scratch((size_t)attn_part_rows(T, (int)B, c.heads, group, (int)max_new, max_kv, window), c.D)});
}

lora_status lora_paged_attn_fwd(const lora_bf16* q, const lora_kv_cache* cache, const int32_t* table, const int32_t* offsets, const int32_t* kv_lens,
                                int64_t T, int32_t H, int64_t B, int64_t max_pages, int64_t ldq, int64_t ldt, int64_t ldo, int64_t max_new,
                                int64_t max_kv, float scale, int32_t window, lora_bf16* out, void* workspace, size_t workspace_bytes,
                                lora_stream stream) {
    AttnArgs a{};
    lora_status st = paged(cache, a.c);
    if (st == LORA_OK) st = check_attn(a.c, T, H, B, max_new, max_kv, window);
    if (st != LORA_OK) return st;
    if (max_pages < 0 || ldt < max_pages) return LORA_ERR_SHAPE;
    if (!(scale > 0.f) || !isfinite(scale)) return LORA_ERR_PARAM;
    if (T == 0 || B == 0 || max_new == 0) return LORA_OK;
    if (!q || !offsets || !kv_lens || !out || !workspace || (max_pages && !table)) return LORA_ERR_NULL;
    if (bad_stride(ldq, H, a.c.D) || bad_stride(ldo, H, a.c.D)) return LORA_ERR_SHAPE;
    if (misaligned(q) || misaligned(out) || misaligned(workspace, 256) || misaligned(table, 4) || misaligned(offsets, 4) || misaligned(kv_lens, 4))
        return LORA_ERR_ALIGN;
    if (max_pages >= 1ll << (30 - a.c.page_shift)) return LORA_ERR_UNSUPPORTED;
    const AttnPlan pl = plan_attn((int)B, a.c.heads, H / a.c.heads, a.c.D, (int)max_new, max_kv, window);
    if ((max_new * (H / a.c.heads) / pl.rows + 1) * pl.splits * B * a.c.heads >= 1ll << 24) return LORA_ERR_UNSUPPORTED;     // (threads of a launch)
    if (workspace_bytes < attn_scratch(pl, T, H, a.c.D)) return LORA_ERR_WORKSPACE;
    a.q = q;
    a.out = out;
    a.table = table;
    a.offsets = offsets;
    a.kv_lens = kv_lens;
    a.part_o = (float*)workspace;
    a.part_ml = (float*)((char*)workspace + align_up((size_t)pl.splits * T * H * a.c.D * 4));
    a.ldq = ldq;
    a.ldo = ldo;
    a.ldt = ldt;
    a.T = (int)T;
    a.B = (int)B;
    a.H = H;
    a.group = H / a.c.heads;
    a.max_pages = (int)max_pages;
    a.window = window;
    a.scale = scale * 1.4426950408889634f;
    return done(launch_attn(a, pl, (int)max_new, (hipStream_t)stream));
}

}  // extern "C"
