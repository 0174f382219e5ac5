// The paged cache of latent vectors (cospec_latent_cache): arguments of its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace cospec {

constexpr int kRotated = 64;          // components of the shared rotated key

// The attentions take a latent cache as PageArgs of one head: k the latents, v the rotated keys, k_scale the
// positions' scales, D the latents' components.
struct LatentAppendArgs {
    PageArgs c;
    const int32_t *start, *count, *positions;
    const char *x, *k_r, *q, *weight;   // bf16
    int64_t ld_c, ld_r, ld_q, head_q, head_out;   // elements
    const float *inv_freq;
    float eps;
    int32_t rot, interleaved, B, n, Hq;
    char *q_out, *c_out, *k_out;
    FastDiv by_n;              // set by the launch
};

// An attention call.  A unit is a block of a sequence's rows; units are numbered by sequence.
struct LatentArgs : PagedArgs {
    int32_t whole;             // the first units, that are not cut
};

// How a call's units are dealt: rounds of one for every CU, and the rest cut into pieces that fill a last round.
struct LatentPlan {
    int32_t rows;              // of a unit, at most
    int32_t blocks;            // units of a sequence
    int64_t units, whole;
    int32_t splits;            // pieces of the units that are cut
    int64_t grid;              // workgroups
    int64_t parts;             // rows of pieces: workspace for {max, sum} and sums each
};

// Query rows of the expanded form, whose keys and values are not paged.
struct ExpandedArgs {
    const char *q, *k, *v, *k_r;        // bf16
    int64_t ld_k, head_k, ld_v, head_v, ld_r;     // elements
    const int32_t *ctx_len, *q_start;
    int32_t B, n_q, L, H, d, K;
    float scale;
    char *out;
    int32_t heads_each;                 // of an XCD; this and the rest set by the launch
    FastDiv by_together, by_blocks, by_heads;
};

hipError_t launch_latent_append(LatentAppendArgs a, hipStream_t s);
hipError_t launch_latent_keep(const KeepArgs &a, hipStream_t s);
LatentPlan latent_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq);
hipError_t launch_latent_attention(LatentArgs a, const LatentPlan &p, hipStream_t s);
int64_t expanded_workgroups(int32_t B, int32_t n_q, int32_t H);
hipError_t launch_expanded_attention(ExpandedArgs a, hipStream_t s);

}  // namespace cospec
