// C ABI of the paged cache of latent vectors, its attentions and the pages under the caches: host-side
// checks and launches.  Declared in include/cospec.h.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "cospec.h"
#include "latent.h"
#include "pages.h"

using namespace cospec;

namespace {

constexpr size_t kAlign = 256;

inline size_t round_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool given(const void *p, size_t a) { return p && aligned(p, a); }

inline bool page_size(int32_t page) { return page == 16 || page == 32 || page == 64 || page == 128; }

inline int32_t log_of(int32_t page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7; }

// Sizes and types of a latent cache (its memory aside).
cospec_status check_latent_sizes(const cospec_latent_cache *c) {
    if (!c || c->n_pages < 0 || c->max_pages < 0) return COSPEC_ERR_INVALID_ARG;
    if (c->dtype != COSPEC_BF16 && c->dtype != COSPEC_F8E4M3) return COSPEC_ERR_UNSUPPORTED;
    if (!page_size(c->page) || (c->d_c != 256 && c->d_c != 512)) return COSPEC_ERR_UNSUPPORTED;
    // pages and a sequence's positions are counted in 32 bits, with room to spare
    if (c->n_pages > INT32_MAX / 4 || c->max_pages > (INT32_MAX - 65536) / c->page) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

cospec_status check_latent(const cospec_latent_cache *c) {
    const cospec_status st = check_latent_sizes(c);
    if (st != COSPEC_OK) return st;
    if (c->n_pages == 0 || c->max_pages == 0) return COSPEC_ERR_INVALID_ARG;
    if (!given(c->c, 16) || !given(c->r, 16) || !given(c->table, 4)) return COSPEC_ERR_INVALID_ARG;
    if (c->dtype == COSPEC_F8E4M3 && !given(c->scale, 4)) return COSPEC_ERR_INVALID_ARG;
    return COSPEC_OK;
}

PageArgs latent_args(const cospec_latent_cache *c) {
    PageArgs p{};
    p.k = static_cast<char *>(c->c); p.v = static_cast<char *>(c->r);
    p.k_scale = c->scale; p.v_scale = nullptr;
    p.table = c->table; p.n_pages = c->n_pages; p.max_pages = c->max_pages;
    p.log_page = log_of(c->page);
    p.H = 1; p.D = c->d_c; p.f8 = c->dtype == COSPEC_F8E4M3;
    return p;
}

// Sizes of an attention call over the cache (0 rows: nothing to do).
cospec_status check_attention_sizes(const cospec_latent_cache *c, int32_t B, int32_t n_q, int32_t Hq) {
    const cospec_status st = check_latent_sizes(c);
    if (st != COSPEC_OK) return st;
    if (B < 0 || n_q < 0 || Hq < 1) return COSPEC_ERR_INVALID_ARG;
    const int64_t wide = static_cast<int64_t>(n_q) * Hq;
    if (wide > INT32_MAX || (wide > 0 && B > INT32_MAX / wide)) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

// The pieces' sums, then their {max, weight sum} pairs.
size_t sums_bytes(const LatentPlan &p, int32_t D) { return round_up(static_cast<size_t>(p.parts) * static_cast<size_t>(D) * 4); }

size_t plan_bytes(const LatentPlan &p, int32_t D) {
    return p.parts == 0 ? 0 : sums_bytes(p, D) + round_up(static_cast<size_t>(p.parts) * 8);
}

cospec_status attend(LatentArgs &a, const cospec_latent_cache *cache, void *workspace, size_t workspace_bytes,
                     hipStream_t stream) {
    const cospec_status st = check_latent(cache);
    if (st != COSPEC_OK) return st;
    if (!given(a.q, 16) || !given(a.out, 16) || !given(a.ctx_len, 4)) return COSPEC_ERR_INVALID_ARG;
    a.c = latent_args(cache);
    const LatentPlan p = latent_plan(a.c, a.B, a.n_q, a.Hq);
    if (p.grid > kMaxWorkgroups / 2) return COSPEC_ERR_UNSUPPORTED;
    if (p.parts > 0) {
        if (!given(workspace, kAlign) || workspace_bytes < plan_bytes(p, a.c.D)) return COSPEC_ERR_WORKSPACE;
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + sums_bytes(p, a.c.D));
    }
    return launch_latent_attention(a, p, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status check_pool(const cospec_page_pool *pool) {
    if (!pool || pool->n_pages < 1 || !given(pool->refs, 4)) return COSPEC_ERR_INVALID_ARG;
    if (!page_size(pool->page) || pool->n_pages > INT32_MAX / 4) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

// Sizes of tables of a pool.
cospec_status check_table(const cospec_page_pool *pool, int32_t rows, int32_t max_pages) {
    const cospec_status st = check_pool(pool);
    if (st != COSPEC_OK) return st;
    if (rows < 0 || max_pages < 1) return COSPEC_ERR_INVALID_ARG;
    if (max_pages > (INT32_MAX - 65536) / pool->page || (rows > 0 && max_pages > INT32_MAX / rows)) return COSPEC_ERR_UNSUPPORTED;
    return COSPEC_OK;
}

}  // namespace

extern "C" {

cospec_status cospec_latent_append(const cospec_latent_cache *cache, const int32_t *start, const int32_t *count,
                                   const void *c, int64_t ld_c, const void *k_r, int64_t ld_r, const void *weight,
                                   float eps, const cospec_rope *rope, const int32_t *positions, int32_t B, int32_t n,
                                   const void *q, int64_t ld_q, int64_t head_q, int32_t Hq, void *q_out,
                                   int64_t head_out, void *c_out, void *k_out, hipStream_t stream) {
    cospec_status st = check_latent_sizes(cache);
    if (st != COSPEC_OK) return st;
    if (B < 0 || n < 0 || (q && Hq < 1) || !isfinite(eps) || eps < 0.f) return COSPEC_ERR_INVALID_ARG;
    LatentAppendArgs a{};
    if (rope) {
        if (rope->rot < 0 || rope->rot > kRotated) return COSPEC_ERR_INVALID_ARG;
        if (rope->rot % 16 != 0) return COSPEC_ERR_UNSUPPORTED;
        if (rope->rot > 0 && !given(rope->inv_freq, 4)) return COSPEC_ERR_INVALID_ARG;
        a.rot = rope->rot;
        a.interleaved = rope->interleaved != 0;
        a.inv_freq = rope->inv_freq;
    }
    if (ld_c < cache->d_c || ld_r < kRotated || ld_c % 8 != 0 || ld_r % 8 != 0) return COSPEC_ERR_INVALID_ARG;
    if (q && (ld_q < 0 || ld_q % 8 != 0 || head_q < kRotated || head_q % 8 != 0 || head_out < kRotated || head_out % 8 != 0))
        return COSPEC_ERR_INVALID_ARG;
    if (static_cast<int64_t>(B) * n == 0) return COSPEC_OK;
    if ((st = check_latent(cache)) != COSPEC_OK) return st;
    if (!given(c, 16) || !given(k_r, 16) || !given(start, 4) || (count && !aligned(count, 4)) ||
        (positions && !aligned(positions, 4)) || (weight && !aligned(weight, 16)) ||
        (q && (!aligned(q, 16) || !given(q_out, 16))) || (c_out && !aligned(c_out, 16)) || (k_out && !aligned(k_out, 16)))
        return COSPEC_ERR_INVALID_ARG;
    const int64_t tokens = static_cast<int64_t>(B) * n;
    if (tokens > kMaxWorkgroups || (q && Hq > INT32_MAX / 1024)) return COSPEC_ERR_UNSUPPORTED;
    a.c = latent_args(cache);
    a.start = start; a.count = count; a.positions = positions;
    a.x = static_cast<const char *>(c); a.k_r = static_cast<const char *>(k_r); a.q = static_cast<const char *>(q);
    a.weight = static_cast<const char *>(weight);
    a.ld_c = ld_c; a.ld_r = ld_r; a.ld_q = ld_q; a.head_q = head_q; a.head_out = head_out;
    a.eps = eps;
    a.B = B; a.n = n; a.Hq = Hq;
    a.q_out = static_cast<char *>(q_out); a.c_out = static_cast<char *>(c_out); a.k_out = static_cast<char *>(k_out);
    return launch_latent_append(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status cospec_latent_keep(const cospec_latent_cache *cache, const int32_t *ctx_len, const int32_t *path,
                                 int32_t B, int32_t N, hipStream_t stream) {
    cospec_status st = check_latent_sizes(cache);
    if (st != COSPEC_OK) return st;
    if (B < 0 || N < 1) return COSPEC_ERR_INVALID_ARG;
    if (N > COSPEC_MAX_N || B > kMaxWorkgroups) return COSPEC_ERR_UNSUPPORTED;
    if (B == 0) return COSPEC_OK;
    if ((st = check_latent(cache)) != COSPEC_OK) return st;
    if (!given(ctx_len, 4) || !given(path, 4)) return COSPEC_ERR_INVALID_ARG;
    KeepArgs a{};
    a.c = latent_args(cache);
    a.ctx_len = ctx_len; a.path = path; a.B = B; a.N = N;
    return launch_latent_keep(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

size_t cospec_latent_attention_workspace_size(const cospec_latent_cache *cache, int32_t B, int32_t n_q, int32_t Hq) {
    if (check_attention_sizes(cache, B, n_q, Hq) != COSPEC_OK) return 0;
    return plan_bytes(latent_plan(latent_args(cache), B, n_q, Hq), cache->d_c);
}

cospec_status cospec_latent_attention(const void *q, const cospec_latent_cache *cache, const int32_t *ctx_len,
                                      const int32_t *q_start, int32_t B, int32_t n_q, int32_t Hq, int32_t K, float scale,
                                      void *out, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!isfinite(scale) || K < 0) return COSPEC_ERR_INVALID_ARG;
    const cospec_status st = check_attention_sizes(cache, B, n_q, Hq);
    if (st != COSPEC_OK) return st;
    if (static_cast<int64_t>(B) * n_q == 0) return COSPEC_OK;
    if (!given(q_start, 4)) return COSPEC_ERR_INVALID_ARG;
    LatentArgs a{};
    a.q = q; a.ctx_len = ctx_len; a.q_start = q_start; a.B = B; a.n_q = n_q; a.Hq = Hq; a.K = K;
    a.scale = scale; a.out = out;
    return attend(a, cache, workspace, workspace_bytes, stream);
}

cospec_status cospec_latent_tree_attention(const void *q, const cospec_latent_cache *cache, const int32_t *ctx_len,
                                           const int32_t *parent, int32_t B, int32_t N, int32_t Hq, float scale,
                                           void *out, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!isfinite(scale) || N < 1) return COSPEC_ERR_INVALID_ARG;
    const cospec_status st = check_attention_sizes(cache, B, N, Hq);
    if (st != COSPEC_OK) return st;
    if (N > COSPEC_MAX_N) return COSPEC_ERR_UNSUPPORTED;
    if (B == 0) return COSPEC_OK;
    if (!given(parent, 4)) return COSPEC_ERR_INVALID_ARG;
    LatentArgs a{};
    a.q = q; a.ctx_len = ctx_len; a.parent = parent; a.B = B; a.n_q = N; a.Hq = Hq;
    a.scale = scale; a.out = out;
    return attend(a, cache, workspace, workspace_bytes, stream);
}

cospec_status cospec_expanded_attention(const void *q, const void *k, int64_t ld_k, int64_t head_k, const void *v,
                                        int64_t ld_v, int64_t head_v, const void *k_r, int64_t ld_r,
                                        const int32_t *ctx_len, const int32_t *q_start, int32_t B, int32_t n_q,
                                        int32_t L, int32_t H, int32_t d, int32_t K, float scale, void *out,
                                        hipStream_t stream) {
    if (!isfinite(scale) || K < 0 || B < 0 || n_q < 0 || L < 0 || H < 1) return COSPEC_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return COSPEC_ERR_UNSUPPORTED;
    if (head_k < d || head_v < d || ld_k < 0 || ld_v < 0 || ld_r < kRotated || (head_k | head_v | ld_k | ld_v | ld_r) % 8 != 0)
        return COSPEC_ERR_INVALID_ARG;
    if (static_cast<int64_t>(B) * n_q == 0) return COSPEC_OK;
    if (!given(q, 16) || !given(out, 16) || !given(ctx_len, 4) || !given(q_start, 4)) return COSPEC_ERR_INVALID_ARG;
    if (L > 0 && (!given(k, 16) || !given(v, 16) || !given(k_r, 16))) return COSPEC_ERR_INVALID_ARG;
    if (static_cast<int64_t>(B) * H > kMaxWorkgroups / 2 || n_q > INT32_MAX - 65536 || L > INT32_MAX - 65536 ||
        expanded_workgroups(B, n_q, H) > kMaxWorkgroups / 2)
        return COSPEC_ERR_UNSUPPORTED;
    ExpandedArgs a{};
    a.q = static_cast<const char *>(q); a.k = static_cast<const char *>(k); a.v = static_cast<const char *>(v);
    a.k_r = static_cast<const char *>(k_r);
    a.ld_k = ld_k; a.head_k = head_k; a.ld_v = ld_v; a.head_v = head_v; a.ld_r = ld_r;
    a.ctx_len = ctx_len; a.q_start = q_start;
    a.B = B; a.n_q = n_q; a.L = L; a.H = H; a.d = d; a.K = K;
    a.scale = scale; a.out = static_cast<char *>(out);
    return launch_expanded_attention(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status cospec_pages_fork(const cospec_page_pool *pool, const int32_t *table, int32_t rows, const int32_t *row,
                                const int32_t *len, int32_t B, int32_t max_pages, int32_t *table_to,
                                hipStream_t stream) {
    cospec_status st = check_table(pool, rows, max_pages);
    if (st == COSPEC_OK) st = check_table(pool, B, max_pages);
    if (st != COSPEC_OK) return st;
    if (B == 0) return COSPEC_OK;
    if ((rows > 0 && !given(table, 4)) || !given(row, 4) || !given(len, 4) || !given(table_to, 4)) return COSPEC_ERR_INVALID_ARG;
    ForkArgs a{};
    a.refs = pool->refs; a.n_pages = pool->n_pages; a.log_page = log_of(pool->page);
    a.table = table; a.rows = rows; a.row = row; a.len = len; a.B = B; a.max_pages = max_pages; a.table_to = table_to;
    return launch_pages_fork(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

size_t cospec_pages_reserve_workspace_size(const cospec_page_pool *pool, int32_t B, int32_t n) {
    if (!pool || !page_size(pool->page) || B < 0 || n < 0) return 0;
    const int64_t touched = pages_touched(n, log_of(pool->page));
    if (B > 0 && touched > INT32_MAX / 4 / B) return 0;
    return 2 * round_up(static_cast<size_t>(std::max<int64_t>(B * touched, 1)) * 4);
}

cospec_status cospec_pages_reserve(const cospec_page_pool *pool, int32_t *table, int32_t max_pages, const int32_t *start,
                                   const int32_t *count, int32_t B, int32_t n, int32_t *copies, int32_t *lacking,
                                   void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const cospec_status st = check_table(pool, B, max_pages);
    if (st != COSPEC_OK) return st;
    if (n < 0 || !given(lacking, 4) || (count && !aligned(count, 4))) return COSPEC_ERR_INVALID_ARG;
    if (B > 0 && (!given(table, 4) || !given(start, 4) || !given(copies, 8))) return COSPEC_ERR_INVALID_ARG;
    const size_t need = cospec_pages_reserve_workspace_size(pool, B, n);
    if (need == 0) return COSPEC_ERR_UNSUPPORTED;
    if (!given(workspace, kAlign) || workspace_bytes < need) return COSPEC_ERR_WORKSPACE;
    ReserveArgs a{};
    a.refs = pool->refs; a.n_pages = pool->n_pages; a.log_page = log_of(pool->page);
    a.table = table; a.max_pages = max_pages; a.start = start; a.count = count; a.B = B; a.n = n;
    a.touched = static_cast<int32_t>(pages_touched(n, a.log_page));
    a.copies = copies; a.lacking = lacking;
    a.rank = static_cast<int32_t *>(workspace);
    a.fresh = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + need / 2);
    return launch_pages_reserve(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status cospec_pages_release(const cospec_page_pool *pool, int32_t *table, int32_t max_pages, const int32_t *keep,
                                   int32_t B, hipStream_t stream) {
    const cospec_status st = check_table(pool, B, max_pages);
    if (st != COSPEC_OK) return st;
    if (B == 0) return COSPEC_OK;
    if (!given(table, 4) || !given(keep, 4)) return COSPEC_ERR_INVALID_ARG;
    ReleaseArgs a{};
    a.refs = pool->refs; a.n_pages = pool->n_pages; a.log_page = log_of(pool->page);
    a.table = table; a.max_pages = max_pages; a.keep = keep; a.B = B;
    return launch_pages_release(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

size_t cospec_pages_compact_workspace_size(const cospec_page_pool *pool) {
    if (!pool || pool->n_pages < 1 || pool->n_pages > INT32_MAX / 4) return 0;
    return round_up(static_cast<size_t>(pool->n_pages) * 4);
}

cospec_status cospec_pages_compact(const cospec_page_pool *pool, int32_t *table, int32_t max_pages, int32_t B,
                                   int32_t *moves, int32_t *n_moves, void *workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
    const cospec_status st = check_table(pool, B, max_pages);
    if (st != COSPEC_OK) return st;
    if ((B > 0 && !given(table, 4)) || !given(moves, 8) || !given(n_moves, 4)) return COSPEC_ERR_INVALID_ARG;
    if (!given(workspace, kAlign) || workspace_bytes < cospec_pages_compact_workspace_size(pool)) return COSPEC_ERR_WORKSPACE;
    CompactArgs a{};
    a.refs = pool->refs; a.n_pages = pool->n_pages;
    a.table = table; a.entries = static_cast<int64_t>(B) * max_pages;
    a.moves = reinterpret_cast<int2 *>(moves); a.n_moves = n_moves;
    a.to = static_cast<int32_t *>(workspace);
    return launch_pages_compact(a, stream) == hipSuccess ? COSPEC_OK : COSPEC_ERR_HIP;
}

cospec_status cospec_pages_copy(const cospec_page_plane *planes, int32_t n_planes, int64_t n_pages,
                                const int32_t *pairs, int32_t n_pairs, const int32_t *count, hipStream_t stream) {
    if (n_planes < 0 || n_pairs < 0 || n_pages < 1 || (n_planes > 0 && !planes)) return COSPEC_ERR_INVALID_ARG;
    if (n_pages > INT32_MAX / 4) return COSPEC_ERR_UNSUPPORTED;
    for (int32_t p = 0; p < n_planes; ++p) {
        if (!given(planes[p].data, 4) || planes[p].page_bytes < 4 || planes[p].page_bytes % 4 != 0) return COSPEC_ERR_INVALID_ARG;
        if (planes[p].page_bytes > (static_cast<int64_t>(1) << 32)) return COSPEC_ERR_UNSUPPORTED;
    }
    if (n_planes == 0 || n_pairs == 0) return COSPEC_OK;
    if (!given(pairs, 8) || (count && !aligned(count, 4))) return COSPEC_ERR_INVALID_ARG;
    for (int32_t first = 0; first < n_planes; first += kMaxPlanes) {
        CopyArgs a{};
        a.n_pages = n_pages; a.pairs = reinterpret_cast<const int2 *>(pairs); a.n_pairs = n_pairs; a.count = count;
        a.n_planes = std::min(n_planes - first, kMaxPlanes);
        for (int p = 0; p < a.n_planes; ++p) {
            a.data[p] = static_cast<char *>(planes[first + p].data);
            a.bytes[p] = planes[first + p].page_bytes;
        }
        if (launch_pages_copy(a, stream) != hipSuccess) return COSPEC_ERR_HIP;
    }
    return COSPEC_OK;
}

}  // extern "C"
