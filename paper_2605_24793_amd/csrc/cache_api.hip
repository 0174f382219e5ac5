// C ABI of the paged key/value cache and its attentions: host-side checks and launches.
// Declared in include/cospec.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cospec.h"
#include "paged.h"

using namespace cospec;

namespace {

constexpr size_t kAlign = 256;

inline size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool given(const void *p, size_t a) { return p && aligned(p, a); }

// Sizes and types of a cache (its memory aside).
cospec_status check_cache_sizes(const cospec_cache *c) {
    if (!c || c->heads < 1 || c->n_pages < 0 || c->max_pages < 0) return COSPEC_ERR_INVALID_ARG;
    if (c->dtype != COSPEC_BF16 && c->dtype != COSPEC_F8E4M3) return COSPEC_ERR_UNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return COSPEC_ERR_UNSUPPORTED;
    if (c->d != 64 && c->d != 128) return COSPEC_ERR_UNSUPPORTED;
    // pages times heads and a sequence's positions are counted in 32 bits, with room to spare
    if (c->n_pages > INT32_MAX / 4 / c->heads || c->max_pages > (INT32_MAX - 65536) / c->page) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

cospec_status check_cache(const cospec_cache *c) {
    const cospec_status st = check_cache_sizes(c);
    if (st != COSPEC_OK) return st;
    if (c->n_pages == 0 || c->max_pages == 0) return COSPEC_ERR_INVALID_ARG;
    if (!given(c->k, 16) || !given(c->v, 16) || !given(c->table, 4)) return COSPEC_ERR_INVALID_ARG;
    if (c->dtype == COSPEC_F8E4M3 && (!given(c->k_scale, 4) || !given(c->v_scale, 4))) return COSPEC_ERR_INVALID_ARG;
    return COSPEC_OK;
}

PageArgs page_args(const cospec_cache *c) {
    PageArgs p{};
    p.k = static_cast<char *>(c->k); p.v = static_cast<char *>(c->v);
    p.k_scale = c->k_scale; p.v_scale = c->v_scale;
    p.table = c->table; p.n_pages = c->n_pages; p.max_pages = c->max_pages;
    p.log_page = c->page == 16 ? 4 : c->page == 32 ? 5 : c->page == 64 ? 6 : 7;
    p.H = c->heads; p.D = c->d; p.f8 = c->dtype == COSPEC_F8E4M3;
    return p;
}

// Sizes of an attention call over the cache (0 rows: nothing to do).
cospec_status check_attention_sizes(const cospec_cache *c, int32_t B, int32_t n_q, int32_t Hq) {
    const cospec_status st = check_cache_sizes(c);
    if (st != COSPEC_OK) return st;
    if (B < 0 || n_q < 0 || Hq < 1 || Hq % c->heads != 0) return COSPEC_ERR_INVALID_ARG;
    const int64_t wide = static_cast<int64_t>(n_q) * Hq;
    if (wide > INT32_MAX || (wide > 0 && B > INT32_MAX / wide)) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

// The pieces' sums, then their {max, weight sum} pairs.
size_t sums_bytes(const PagedPlan &p, int32_t D) {
    return round_up(static_cast<size_t>(p.splits) * static_cast<size_t>(p.rows) * static_cast<size_t>(D) * 4);
}

size_t plan_bytes(const PagedPlan &p, int32_t D) {
    if (p.splits < 2) return 0;
    return sums_bytes(p, D) + round_up(static_cast<size_t>(p.splits) * static_cast<size_t>(p.rows) * 8);
}

cospec_status attend(PagedArgs &a, const cospec_cache *cache, void *workspace, size_t workspace_bytes,
                     hipStream_t stream) {
    const cospec_status st = check_cache(cache);
    if (st != COSPEC_OK) return st;
    if (!given(a.q, 16) || !given(a.out, 16) || !given(a.ctx_len, 4)) return COSPEC_ERR_INVALID_ARG;
    a.c = page_args(cache);
    const PagedPlan p = paged_plan(a.c, a.B, a.n_q, a.Hq);
    if (p.grid > kMaxWorkgroups) return COSPEC_ERR_UNSUPPORTED;
    if (p.splits > 1) {
        if (!given(workspace, kAlign) || workspace_bytes < plan_bytes(p, a.c.D)) return COSPEC_ERR_WORKSPACE;
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + sums_bytes(p, a.c.D));
    }
    return launch_paged_attention(a, p, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

}  // namespace

extern "C" {

cospec_status cospec_cache_append(const cospec_cache *cache, const int32_t *start, const int32_t *count,
                                  const void *k, int64_t ld_k, const void *v, int64_t ld_v,
                                  const cospec_rope *rope, const int32_t *positions, int32_t B, int32_t n,
                                  const void *q, int64_t ld_q, int32_t Hq, void *q_out, hipStream_t stream) {
    cospec_status st = check_cache_sizes(cache);
    if (st != COSPEC_OK) return st;
    if (B < 0 || n < 0 || (q && Hq < 1)) return COSPEC_ERR_INVALID_ARG;
    AppendArgs a{};
    if (rope) {
        if (rope->rot < 0 || rope->rot > cache->d) return COSPEC_ERR_INVALID_ARG;
        if (rope->rot % 16 != 0) return COSPEC_ERR_UNSUPPORTED;
        if (rope->rot > 0 && !given(rope->inv_freq, 4)) return COSPEC_ERR_INVALID_ARG;
        a.rot = rope->rot;
        a.interleaved = rope->interleaved != 0;
        a.inv_freq = rope->inv_freq;
    }
    const int64_t row = static_cast<int64_t>(cache->heads) * cache->d;
    if (ld_k < row || ld_v < row || ld_k % 8 != 0 || ld_v % 8 != 0) return COSPEC_ERR_INVALID_ARG;
    if (q && (ld_q < static_cast<int64_t>(Hq) * cache->d || ld_q % 8 != 0)) return COSPEC_ERR_INVALID_ARG;
    if (static_cast<int64_t>(B) * n == 0) return COSPEC_OK;
    if ((st = check_cache(cache)) != COSPEC_OK) return st;
    if (!given(k, 16) || !given(v, 16) || !given(start, 4) || (count && !aligned(count, 4)) ||
        (positions && !aligned(positions, 4)) || (q && (!aligned(q, 16) || !given(q_out, 16))))
        return COSPEC_ERR_INVALID_ARG;
    a.c = page_args(cache);
    const int64_t per_sequence = pages_touched(n, a.c.log_page) * cache->heads;
    const int64_t query_groups = q ? (static_cast<int64_t>(B) * n + kQueryTokens - 1) / kQueryTokens : 0;
    if (static_cast<int64_t>(B) * n > INT32_MAX / 2 || per_sequence > kMaxWorkgroups / B ||
        per_sequence * B + query_groups > kMaxWorkgroups || static_cast<int64_t>(Hq) * cache->d > INT32_MAX / 16)
        return COSPEC_ERR_UNSUPPORTED;
    a.start = start; a.count = count; a.positions = positions;
    a.k = static_cast<const char *>(k); a.v = static_cast<const char *>(v); a.q = static_cast<const char *>(q);
    a.ld_k = ld_k; a.ld_v = ld_v; a.ld_q = ld_q;
    a.B = B; a.n = n; a.Hq = Hq;
    a.q_out = static_cast<char *>(q_out);
    return launch_cache_append(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status cospec_cache_keep(const cospec_cache *cache, const int32_t *ctx_len, const int32_t *path, int32_t B,
                                int32_t N, hipStream_t stream) {
    cospec_status st = check_cache_sizes(cache);
    if (st != COSPEC_OK) return st;
    if (B < 0 || N < 1) return COSPEC_ERR_INVALID_ARG;
    if (N > COSPEC_MAX_N || cache->heads > kMaxWorkgroups / 2 / (B > 0 ? B : 1)) return COSPEC_ERR_UNSUPPORTED;
    if (B == 0) return COSPEC_OK;
    if ((st = check_cache(cache)) != COSPEC_OK) return st;
    if (!given(ctx_len, 4) || !given(path, 4)) return COSPEC_ERR_INVALID_ARG;
    KeepArgs a{};
    a.c = page_args(cache);
    a.ctx_len = ctx_len; a.path = path; a.B = B; a.N = N;
    return launch_cache_keep(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

size_t cospec_paged_attention_workspace_size(const cospec_cache *cache, int32_t B, int32_t n_q, int32_t Hq) {
    if (check_attention_sizes(cache, B, n_q, Hq) != COSPEC_OK) return 0;
    return plan_bytes(paged_plan(page_args(cache), B, n_q, Hq), cache->d);
}

cospec_status cospec_hybrid_attention_paged(const void *q, const cospec_cache *cache, const int32_t *ctx_len,
                                            const int32_t *q_start, int32_t B, int32_t n_q, int32_t Hq, int32_t K,
                                            float scale, void *out, void *workspace, size_t workspace_bytes,
                                            hipStream_t stream) {
    if (!isfinite(scale) || K < 0) return COSPEC_ERR_INVALID_ARG;
    const cospec_status st = check_attention_sizes(cache, B, n_q, Hq);
    if (st != COSPEC_OK) return st;
    if (static_cast<int64_t>(B) * n_q == 0) return COSPEC_OK;
    if (!given(q_start, 4)) return COSPEC_ERR_INVALID_ARG;
    PagedArgs a{};
    a.q = q; a.ctx_len = ctx_len; a.q_start = q_start; a.B = B; a.n_q = n_q; a.Hq = Hq; a.K = K;
    a.scale = scale; a.out = out;
    return attend(a, cache, workspace, workspace_bytes, stream);
}

cospec_status cospec_tree_attention(const void *q, const cospec_cache *cache, const int32_t *ctx_len,
                                    const int32_t *parent, int32_t B, int32_t N, int32_t Hq, float scale, void *out,
                                    void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!isfinite(scale) || N < 1) return COSPEC_ERR_INVALID_ARG;
    const cospec_status st = check_attention_sizes(cache, B, N, Hq);
    if (st != COSPEC_OK) return st;
    if (N > COSPEC_MAX_N) return COSPEC_ERR_UNSUPPORTED;
    if (B == 0) return COSPEC_OK;
    if (!given(parent, 4)) return COSPEC_ERR_INVALID_ARG;
    PagedArgs a{};
    a.q = q; a.ctx_len = ctx_len; a.parent = parent; a.B = B; a.n_q = N; a.Hq = Hq;
    a.scale = scale; a.out = out;
    return attend(a, cache, workspace, workspace_bytes, stream);
}

}  // extern "C"
