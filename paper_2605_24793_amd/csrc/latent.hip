// Writing the paged cache of latent vectors: appending new positions (latents normalised, keys rotated
// to their place, queries' rotated part beside them) and keeping the accepted path of a token
// tree.
//
// 8-bit latents have a power-of-two scale for each position: a scale of a whole page would be tighter
// in memory (4 bytes of 644), but then later tokens would round the earlier ones anew, and a page
// could not be copied or kept position by position.
#include "cache_math.h"
#include "latent.h"

namespace cospec {
namespace {

constexpr int kTokenThreads = 256;
constexpr int kTokensPerGroup = kTokenThreads / 64;

__device__ inline float max_wave(float x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    return x;
}

// One wave per token.  Its lanes hold eight of the latent's components each; sums and products of the
// norm are in double precision (a few instructions a lane), so that a value next to a border of the
// 8-bit type falls where 64 bits put it.
//
// Whole inputs are bound by memory: 4 x 2065 tokens with 32 heads' queries, into bf16 pages and densely, 25.0 us, 3.9 TB/s of
// the 4.7 that a large copy reaches.  One token is a launch: start and table, token, page; 3.9 us of kernel, 5.5 a call.
template <int DC, bool F8, int INTERLEAVED>
__global__ __launch_bounds__(kTokenThreads) void k_latent_append(LatentAppendArgs a) {
    constexpr int LANES = DC / 8;                           // with a part of the latent
    constexpr int PAIRS = kRotated / 2;
    constexpr int UPT = kRotated / 16;                      // units of a head's rotated part
    __shared__ float2 s_cs[kTokensPerGroup][PAIRS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t tok = static_cast<int64_t>(blockIdx.x) * kTokensPerGroup + wave;
    const bool there = tok < static_cast<int64_t>(a.B) * a.n;
    const int64_t t = there ? tok : 0;                      // (waves of no token read the first, and write nothing)
    const int b = quot(a.by_n, static_cast<uint32_t>(t));
    const int i = static_cast<int>(t) - b * a.n;
    const bool part = lane < LANES;
    u32x4 w = {0, 0, 0, 0}, wt = {0, 0, 0, 0}, kw[2] = {};
    if (part) w = *reinterpret_cast<const u32x4 *>(a.x + (t * a.ld_c + lane * 8) * 2);
    const Unit ku = unit_of(lane % UPT, a.rot, INTERLEAVED);
    if (lane < UPT) load_unit(a.k_r + t * a.ld_r * 2, ku, kw);
    if (a.weight && part) wt = *reinterpret_cast<const u32x4 *>(a.weight + lane * 16);
    const int64_t start = a.start[b];
    const int64_t at = start + i;
    const int64_t room = static_cast<int64_t>(a.c.max_pages) << a.c.log_page;
    const int cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const bool kept = there && i < cnt && at >= 0 && at < room;
    int64_t pid = -1;
    if (kept) pid = page_or_none(a.c, a.c.table[static_cast<int64_t>(b) * a.c.max_pages + (at >> a.c.log_page)]);
    if (lane < a.rot / 2)
        s_cs[wave][lane] = turn(a.positions ? a.positions[t] : at, turns_of(a.inv_freq[lane]));
    __syncthreads();                                        // the last one: waves go on alone
    if (!there) return;
    const float2 *cs = s_cs[wave];

    float x[8];
    unpack8(w, x);
    if (a.weight) {
        double ss = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fma(static_cast<double>(x[e]), static_cast<double>(x[e]), ss);
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) ss += __shfl_xor(ss, off);
        const double r = 1.0 / sqrt(ss * (1.0 / DC) + static_cast<double>(a.eps));
        float g[8];
        unpack8(wt, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(static_cast<double>(x[e]) * r * static_cast<double>(g[e]));
    }
    const u32x4 rounded{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    if (a.c_out && part) *reinterpret_cast<u32x4 *>(a.c_out + (t * DC + lane * 8) * 2) = rounded;
    const int64_t place = (pid << a.c.log_page) + (at & ((1 << a.c.log_page) - 1));
    if constexpr (F8) {
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(x[e]));
        const float s = scale_for(max_wave(part ? top : 0.f)), inv = 1.f / s;
        if (pid >= 0) {
            if (part)
                *reinterpret_cast<u32x2 *>(a.c.k + place * DC + lane * 8) =
                    u32x2{f8_quad(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                          f8_quad(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
            if (lane == 0) a.c.k_scale[place] = s;
        }
    } else {
        if (pid >= 0 && part) *reinterpret_cast<u32x4 *>(a.c.k + (place * DC + lane * 8) * 2) = rounded;
    }
    if (lane < UPT) {
        float y[16];
        unpack8(kw[0], y);
        unpack8(kw[1], y + 8);
        if (ku.pair >= 0) {
#pragma unroll
            for (int p = 0; p < 8; ++p) rotate_pair<INTERLEAVED>(y, p, cs[ku.pair + p]);
        }
        if (pid >= 0) store_bf16(a.c.v + place * (kRotated * 2), ku, y);
        if (a.k_out) store_bf16(a.k_out + t * (kRotated * 2), ku, y);
    }
    if (!a.q) return;
#pragma unroll 2
    for (int h = lane / UPT; h < a.Hq; h += 64 / UPT) {
        u32x4 qw[2];
        load_unit(a.q + (t * a.ld_q + h * a.head_q) * 2, ku, qw);
        float y[16];
        unpack8(qw[0], y);
        unpack8(qw[1], y + 8);
        if (ku.pair >= 0) {
#pragma unroll
            for (int p = 0; p < 8; ++p) rotate_pair<INTERLEAVED>(y, p, cs[ku.pair + p]);
        }
        store_bf16(a.q_out + (t * a.Hq + h) * a.head_out * 2, ku, y);
    }
}

// One workgroup per sequence moves its path's positions, sixteen at a time, four of each wave.  A
// batch is read before any of it is written; what a batch writes, no later one reads, as path[i] >= i
// increases.  A launch of a few round trips (path, table, places, write).
template <int DC, bool F8>
__global__ __launch_bounds__(kTokenThreads) void k_latent_keep(KeepArgs a) {
    constexpr int EB = F8 ? 1 : 2;
    constexpr int LANES = DC * EB / 16, EACH = 4;
    __shared__ int s_path[kMaxSeqRows];
    __shared__ int s_end;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    if (tid == 0) s_end = a.N;
    __syncthreads();
    if (tid < a.N) {
        const int p = a.path[static_cast<int64_t>(b) * a.N + tid];
        s_path[tid] = p;
        if (p < 0 || p >= a.N) atomicMin(&s_end, tid);
    }
    __syncthreads();
    const int end = s_end;
    const int64_t lc = max(a.ctx_len[b], 0), room = static_cast<int64_t>(a.c.max_pages) << a.c.log_page;
    auto place_at = [&](int64_t pos) -> int64_t {
        if (pos >= room) return -1;
        const int64_t pid = page_or_none(a.c, a.c.table[static_cast<int64_t>(b) * a.c.max_pages + (pos >> a.c.log_page)]);
        return pid < 0 ? -1 : (pid << a.c.log_page) + (pos & ((1 << a.c.log_page) - 1));
    };
    for (int base = 0; base < end; base += EACH * kTokensPerGroup) {
        int64_t to[EACH];
        u32x4 x[EACH] = {}, r[EACH] = {};
        float s[EACH] = {};
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int i = base + wave * EACH + e;
            to[e] = -1;
            if (i >= end || s_path[i] == i) continue;
            const int64_t from = place_at(lc + s_path[i]);
            if (from < 0) continue;
            to[e] = place_at(lc + i);
            if (lane < LANES) x[e] = *reinterpret_cast<const u32x4 *>(a.c.k + from * (DC * EB) + lane * 16);
            if (lane < 8) r[e] = *reinterpret_cast<const u32x4 *>(a.c.v + from * (kRotated * 2) + lane * 16);
            if (F8) s[e] = a.c.k_scale[from];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            if (to[e] < 0) continue;
            if (lane < LANES) *reinterpret_cast<u32x4 *>(a.c.k + to[e] * (DC * EB) + lane * 16) = x[e];
            if (lane < 8) *reinterpret_cast<u32x4 *>(a.c.v + to[e] * (kRotated * 2) + lane * 16) = r[e];
            if (F8 && lane == 0) a.c.k_scale[to[e]] = s[e];
        }
        __syncthreads();
    }
}

template <int DC, bool F8> void run_append(const LatentAppendArgs &a, dim3 grid, hipStream_t s) {
    if (a.interleaved) hipLaunchKernelGGL((k_latent_append<DC, F8, 1>), grid, dim3(kTokenThreads), 0, s, a);
    else hipLaunchKernelGGL((k_latent_append<DC, F8, 0>), grid, dim3(kTokenThreads), 0, s, a);
}

}  // namespace

hipError_t launch_latent_append(LatentAppendArgs a, hipStream_t s) {
    a.by_n = fast_div(a.n);
    const int64_t tokens = static_cast<int64_t>(a.B) * a.n;
    const dim3 grid(static_cast<unsigned>((tokens + kTokensPerGroup - 1) / kTokensPerGroup));
    if (a.c.D == 512) a.c.f8 ? run_append<512, true>(a, grid, s) : run_append<512, false>(a, grid, s);
    else a.c.f8 ? run_append<256, true>(a, grid, s) : run_append<256, false>(a, grid, s);
    return hipGetLastError();
}

hipError_t launch_latent_keep(const KeepArgs &a, hipStream_t s) {
    const dim3 grid(a.B), t(kTokenThreads);
    if (a.c.D == 512) {
        if (a.c.f8) hipLaunchKernelGGL((k_latent_keep<512, true>), grid, t, 0, s, a);
        else hipLaunchKernelGGL((k_latent_keep<512, false>), grid, t, 0, s, a);
    } else {
        if (a.c.f8) hipLaunchKernelGGL((k_latent_keep<256, true>), grid, t, 0, s, a);
        else hipLaunchKernelGGL((k_latent_keep<256, false>), grid, t, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace cospec
