// The paged key/value cache (cospec_cache): arguments of its kernels and what they share.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "launch.h"
#include "paged_ranges.h"

namespace cospec {

// Workgroups of a launch, at most: a grid holds fewer than 2^32 threads, and they have 256.
constexpr int64_t kMaxWorkgroups = (1 << 24) - 1;

// Keys [n_pages][H][P][D], values [n_pages][H][D][P], P = 1 << log_page.
struct PageArgs {
    char *k, *v;
    float *k_scale, *v_scale;  // [n_pages][H], 8-bit pages only
    const int32_t *table;      // [B][max_pages]
    int64_t n_pages;
    int32_t max_pages, log_page, H, D, f8;
};

struct AppendArgs {
    PageArgs c;
    const int32_t *start, *count, *positions;
    const char *k, *v, *q;     // bf16
    int64_t ld_k, ld_v, ld_q;  // elements
    const float *inv_freq;
    int32_t rot, interleaved, B, n, Hq;
    char *q_out;
    // set by the launch: page workgroups ahead of the query ones, and their divisions
    uint32_t page_wgs;
    FastDiv by_pages, by_heads, by_n, by_chunks[9];   // by_chunks: by 1 .. 8, sixteen-place chunks of a page
};

struct KeepArgs {
    PageArgs c;
    const int32_t *ctx_len, *path;
    int32_t B, N;
    FastDiv by_heads;
};

// Queries of a hybrid call (q_start, K) or of tree nodes (parent, n_q = N).
struct PagedArgs {
    PageArgs c;
    const void *q;
    const int32_t *ctx_len, *q_start, *parent;
    int32_t B, n_q, Hq, K;
    float scale;
    void *out;
    // keys cut into at most `splits` pieces: unnormalised sums [splits][rows][D] and {running
    // max, weight sum} [splits][rows], rows = B * n_q * Hq
    int32_t splits;
    float *part_o;
    float2 *part_ml;
    // set by the launch
    int32_t row_tiles, row_waves;   // 16-row tiles of a wave, waves with rows of their own
    int32_t min_piece;         // keys of a piece, at least
    FastDiv by_grp, by_blocks, by_heads, by_splits, by_seq_rows, by_hq;
};

struct PagedPlan {
    int32_t row_tiles, row_waves, blocks, splits, min_piece;   // blocks: workgroups that share a group's rows
    int64_t rows;                        // B * n_q * Hq
    int64_t grid;                        // workgroups
};

// Pages that a sequence's n new positions can touch, wherever they start.
inline int64_t pages_touched(int64_t n, int32_t log_page) { return ((n + (1 << log_page) - 2) >> log_page) + 1; }

// Tokens of a workgroup that rotates queries.  One sequence of 2000 tokens, e4m3: 8 tokens 10.8 us, 4 tokens 12.1, 16 14.9;
// 64 x 17 11.3, 11.1 and 15.5 (as bf16 14.9, 12.8 and 19.2), 64 x 1 7.5, 6.2 and 10.8; 4 x 2065 46.7, 44.6 and 48.4.
constexpr int kQueryTokens = 8;

PagedPlan paged_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq);
hipError_t launch_cache_append(AppendArgs a, hipStream_t s);
hipError_t launch_cache_keep(KeepArgs a, hipStream_t s);
hipError_t launch_paged_attention(PagedArgs a, const PagedPlan &p, hipStream_t s);

// The page a table entry names, or -1.
__device__ inline int64_t page_or_none(const PageArgs &c, int32_t id) {
    return id >= 0 && id < c.n_pages ? id : -1;
}

}  // namespace cospec
