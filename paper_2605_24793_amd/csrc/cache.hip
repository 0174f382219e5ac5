// Writing the paged key/value cache: appending new positions (keys rotated to their place,
// values transposed into the pages' layout, queries rotated beside them) and keeping the
// accepted path of a token tree.
//
// 8-bit pages hold e4m3 values with one power-of-two scale per page and head.  A floating type
// loses nothing to a scale's mantissa, and with powers of two a page whose scale grows keeps its
// earlier values' bits (only the exponents move; what becomes subnormal is rounded once more).
#include <algorithm>

#include "paged.h"

namespace cospec {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kCacheThreads = 256;
constexpr int kMaxPage = 128;
// new tokens of a page whose values are stored one by one: 64 x 1 token 7.5 us so and 8.0 by sixteen
// places, 64 x 4 9.3 and 8.8
constexpr int kFewTokens = 2;
constexpr float kLowestScale = 7.888609052210118e-31f;   // 2^-100

__device__ inline uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Four values -> four e4m3 bytes, round to nearest even, NaN beyond the largest.
__device__ inline uint32_t f8_quad(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

__device__ inline uint32_t f8_byte(float a) {
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(a, a, 0, false)) & 0xffu;
}

__device__ inline float f8_value(uint32_t byte) {
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(byte), 0);
}

// Four e4m3 bytes, each times f (a power of two), rounded anew.
__device__ inline uint32_t f8_rescaled(uint32_t w, float f) {
    const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
    const floatx2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    return f8_quad(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// The smallest power of two s >= 2^-100 with amax <= 448 s: 448 is 1.75 * 2^8.
__device__ inline float scale_for(float amax) {
    const uint32_t w = __float_as_uint(amax);
    const int e = static_cast<int>(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u);
    return e < -100 ? kLowestScale : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// The power of two of a scale (its mantissa bits are not used).
__device__ inline float power_of(float s) { return __uint_as_float(__float_as_uint(s) & 0x7f800000u); }

// cos and sin of 2 pi f, |f| <= 1/2.  The nearest quarter turn is taken off, which leaves x, |x| <= pi / 4,
// for the Taylor sums of sin to x^9 and cos to x^10 (the next terms are below 2e-9 and 2e-10);
// the quarter turns swap them and set the signs.
__device__ inline float2 cos_sin_turns(float f) {
    const float q = rintf(4.f * f);
    const float x = 6.28318530717958648f * fmaf(q, -0.25f, f), z = x * x;
    float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
    s = fmaf(z, s, 8.33333333e-3f);
    s = fmaf(z, s, -1.66666667e-1f);
    s = fmaf(z * x, s, x);
    float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
    c = fmaf(z, c, -1.38888889e-3f);
    c = fmaf(z, c, 4.16666667e-2f);
    c = fmaf(z, c, -0.5f);
    c = fmaf(z, c, 1.f);
    const int n = static_cast<int>(q);
    const float u = n & 1 ? s : c, v = n & 1 ? c : s;
    return make_float2(__uint_as_float(__float_as_uint(u) ^ (((n + 1) & 2) ? 0x80000000u : 0u)),
                       __uint_as_float(__float_as_uint(v) ^ ((n & 2) ? 0x80000000u : 0u)));
}

// Turns of a pair per position, in double precision, and cos and sin at a position: the product is
// reduced to a fraction of a turn in double precision (far positions then lose nothing; the rest,
// sine and cosine of a fraction, is fp32).
__device__ inline double turns_of(float inv_freq) { return static_cast<double>(inv_freq) * 0.15915494309189535; }

__device__ inline float2 turn(int64_t position, double turns) {
    const double t = static_cast<double>(position) * turns;
    return cos_sin_turns(static_cast<float>(t - rint(t)));
}

// max over the workgroup, in every thread; `s` one float per wave, free to reuse only after
// another barrier.
__device__ inline float max_group(float x, float *s) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int w = 1; w < kCacheThreads / 64; ++w) x = fmaxf(x, s[w]);
    return x;
}

__device__ inline float finite_abs(float x) {
    const float a = fabsf(x);
    return a < INFINITY ? a : 0.f;     // false for NaN too
}

// A token's head of D components is handled in units of sixteen: two runs of eight, `a` and `b`,
// that hold the two halves of eight pairs where the unit is rotated.
struct Unit {
    int a, b;      // first component of each run
    int pair;      // first of the eight pairs, or -1: not rotated
};

__device__ inline Unit unit_of(int u, int rot, int interleaved) {
    if (16 * u >= rot) return Unit{16 * u, 16 * u + 8, -1};
    if (interleaved) return Unit{16 * u, 16 * u + 8, 8 * u};
    return Unit{8 * u, rot / 2 + 8 * u, 8 * u};
}

__device__ inline void unpack8(u32x4 w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}

// The unit's sixteen values: run a, then run b.
__device__ inline void load_unit(const char *row, const Unit &u, u32x4 (&w)[2]) {
    w[0] = *reinterpret_cast<const u32x4 *>(row + u.a * 2);
    w[1] = *reinterpret_cast<const u32x4 *>(row + u.b * 2);
}

// Pair i of the unit rotated by t = {cos, sin}.
template <int INTERLEAVED> __device__ inline void rotate_pair(float *x, int i, float2 t) {
    const int p1 = INTERLEAVED ? 2 * i : i, p2 = INTERLEAVED ? 2 * i + 1 : i + 8;
    const float x1 = x[p1], x2 = x[p2];
    x[p1] = x1 * t.x - x2 * t.y;
    x[p2] = x2 * t.x + x1 * t.y;
}

__device__ inline void store_bf16(char *row, const Unit &u, const float *x) {
    *reinterpret_cast<u32x4 *>(row + u.a * 2) =
        u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    *reinterpret_cast<u32x4 *>(row + u.b * 2) =
        u32x4{bf16_pair(x[8], x[9]), bf16_pair(x[10], x[11]), bf16_pair(x[12], x[13]), bf16_pair(x[14], x[15])};
}

// Rotates the queries of kQueryTokens tokens from token t0 on: cos and sin of every token's pairs once,
// for all heads.
template <int D, int INTERLEAVED>
__device__ inline void rotate_queries(const AppendArgs &a, int64_t t0, float2 *s_cs) {
    constexpr int UPT = D / 16;
    const int tid = threadIdx.x, pairs = a.rot / 2;
    const int T = static_cast<int>(min(static_cast<int64_t>(kQueryTokens), static_cast<int64_t>(a.B) * a.n - t0));
    constexpr int TPT = kCacheThreads / kQueryTokens;       // threads of a token
    {
        const int t = tid / TPT;
        if (t < T) {
            const int64_t tok = t0 + t;
            const int b = quot(a.by_n, static_cast<uint32_t>(tok));
            const int64_t pos = a.positions ? a.positions[tok] : a.start[b] + (tok - static_cast<int64_t>(b) * a.n);
            for (int i = tid % TPT; i < pairs; i += TPT) s_cs[t * (D / 2) + i] = turn(pos, turns_of(a.inv_freq[i]));
        }
    }
    __syncthreads();
    const Unit u = unit_of(tid % UPT, a.rot, INTERLEAVED);
    for (int h = tid / UPT; h < a.Hq; h += kCacheThreads / UPT) {
#pragma unroll 4
        for (int t = 0; t < T; ++t) {
            u32x4 w[2];
            load_unit(a.q + ((t0 + t) * a.ld_q + h * D) * 2, u, w);
            float x[16];
            unpack8(w[0], x);
            unpack8(w[1], x + 8);
            if (u.pair >= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) rotate_pair<INTERLEAVED>(x, i, s_cs[t * (D / 2) + u.pair + i]);
            }
            store_bf16(a.q_out + ((t0 + t) * a.Hq + h) * D * 2, u, x);
        }
    }
}

// One workgroup per (sequence, page it touches, head) writes the page's new keys and values,
// or, from workgroup page_wgs on, rotates queries.
//
// Keys: a thread holds its units' rotated values in registers while the workgroup finds their
// largest, so they are read once and rounded once; a thread's units are of the same pairs.  Values:
// staged in LDS as rows, read as columns, since a page holds them transposed; a thread
// writes sixteen places of two components at a time, merged with what the page holds where only
// some of them are new.  The tokens' loads wait for the sequence's start only, not for its page.
template <int D, bool F8, int INTERLEAVED>
__global__ __launch_bounds__(kCacheThreads) void k_cache_append(AppendArgs a) {
    constexpr int UPT = D / 16;                             // units of a token's head
    constexpr int MAXU = kMaxPage * UPT / kCacheThreads;    // units of a thread
    constexpr int EB = F8 ? 1 : 2;
    constexpr int VW = D / 2 + 1;                           // words of a staged value row: odd
    extern __shared__ __attribute__((aligned(16))) char s_dyn[];   // value rows, or the queries' cos and sin
    __shared__ float s_max[2][kCacheThreads / 64];
    const int tid = threadIdx.x;
    if (blockIdx.x >= a.page_wgs) {
        rotate_queries<D, INTERLEAVED>(a, static_cast<int64_t>(blockIdx.x - a.page_wgs) * kQueryTokens,
                                       reinterpret_cast<float2 *>(s_dyn));
        return;
    }
    uint32_t *s_v = reinterpret_cast<uint32_t *>(s_dyn);

    const uint32_t bj = quot(a.by_heads, blockIdx.x);
    const int h = blockIdx.x - bj * a.by_heads.d;
    const int b = quot(a.by_pages, bj);
    const int64_t start = a.start[b];
    const int64_t cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const int64_t j = (max(start, static_cast<int64_t>(0)) >> a.c.log_page) + (bj - b * a.by_pages.d);
    const NewPlaces places = new_places(start, cnt, j, a.c.log_page);
    const int64_t base = places.base;
    const int lo = places.lo, hi = places.hi;
    if (lo >= hi || j >= a.c.max_pages) return;
    const int32_t id = a.c.table[static_cast<int64_t>(b) * a.c.max_pages + j];
    const int T = hi - lo;
    const int64_t tok0 = static_cast<int64_t>(b) * a.n + base + lo;    // row of the first new token
    const Unit u = unit_of(tid % UPT, a.rot, INTERLEAVED);

    u32x4 kw[MAXU][2];
    int64_t pos[MAXU];
    float inv_freq[8] = {};
#pragma unroll
    for (int m = 0; m < MAXU; ++m) {
        const int t = (m * kCacheThreads + tid) / UPT;
        if (t >= T) continue;
        load_unit(a.k + ((tok0 + t) * a.ld_k + h * D) * 2, u, kw[m]);
        pos[m] = a.positions ? a.positions[tok0 + t] : start + base + lo + t;
    }
    if (u.pair >= 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) inv_freq[i] = a.inv_freq[u.pair + i];
    }
    float vmax = 0.f;
    for (int e = tid; e < T * (D / 8); e += kCacheThreads) {
        const int t = e / (D / 8), c8 = e % (D / 8);
        const u32x4 w = *reinterpret_cast<const u32x4 *>(a.v + ((tok0 + t) * a.ld_v + h * D + c8 * 8) * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s_v[t * VW + c8 * 4 + i] = w[i];
            if (F8) vmax = fmaxf(vmax, fmaxf(finite_abs(bf16_lo(w[i])), finite_abs(bf16_hi(w[i]))));
        }
    }
    const int64_t pid = page_or_none(a.c, id);
    if (pid < 0) return;                                    // the whole workgroup
    const int64_t blk = pid * a.c.H + h;
    float k_old = 0.f, v_old = 0.f;                         // scales, where the page holds earlier positions
    if (F8 && lo > 0) {
        k_old = power_of(a.c.k_scale[blk]);
        v_old = power_of(a.c.v_scale[blk]);
    }
    float x[MAXU][16], kmax = 0.f;
#pragma unroll
    for (int m = 0; m < MAXU; ++m) {
        const int t = (m * kCacheThreads + tid) / UPT;
        if (t < T) {
            unpack8(kw[m][0], x[m]);
            unpack8(kw[m][1], x[m] + 8);
            if (u.pair >= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    rotate_pair<INTERLEAVED>(x[m], i, turn(pos[m], turns_of(inv_freq[i])));
            }
            if (F8) {
#pragma unroll
                for (int i = 0; i < 16; ++i) kmax = fmaxf(kmax, finite_abs(x[m][i]));
            }
        }
    }
    float kinv = 1.f, vinv = 1.f, kfac = 1.f, vfac = 1.f;
    if constexpr (F8) {
        const float ks = fmaxf(scale_for(max_group(kmax, s_max[0])), k_old);
        const float vs = fmaxf(scale_for(max_group(vmax, s_max[1])), v_old);
        if (lo > 0) {
            kfac = k_old / ks;
            vfac = v_old / vs;
        }
        kinv = 1.f / ks;
        vinv = 1.f / vs;
        __syncthreads();                                    // every thread has read the present scales
        if (tid == 0) {
            a.c.k_scale[blk] = ks;
            a.c.v_scale[blk] = vs;
        }
    } else {
        __syncthreads();                                    // the value rows are staged
    }
    char *kp = a.c.k + (blk << a.c.log_page) * (D * EB);
#pragma unroll
    for (int m = 0; m < MAXU; ++m) {
        const int t = (m * kCacheThreads + tid) / UPT;
        if (t >= T) continue;
        char *row = kp + static_cast<int64_t>(lo + t) * (D * EB);
        if constexpr (F8) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = f8_quad(x[m][4 * i] * kinv, x[m][4 * i + 1] * kinv, x[m][4 * i + 2] * kinv, x[m][4 * i + 3] * kinv);
            *reinterpret_cast<u32x2 *>(row + u.a) = u32x2{w[0], w[1]};
            *reinterpret_cast<u32x2 *>(row + u.b) = u32x2{w[2], w[3]};
        } else {
            store_bf16(row, u, x[m]);
        }
    }
    if constexpr (F8) {
        if (kfac != 1.f) {
            uint32_t *w = reinterpret_cast<uint32_t *>(kp);
            for (int e = tid; e < lo * (D / 4); e += kCacheThreads) w[e] = f8_rescaled(w[e], kfac);
        }
    }
    char *vp = a.c.v + (blk << a.c.log_page) * (D * EB);
    if (T <= kFewTokens && vfac == 1.f) {                   // an element each, nothing to merge
        for (int e = tid; e < T * D; e += kCacheThreads) {
            const int t = e / D, d = e % D;
            const uint32_t v = s_v[t * VW + d / 2];
            const int64_t at = (static_cast<int64_t>(d) << a.c.log_page) + lo + t;
            if constexpr (F8) vp[at] = static_cast<char>(f8_byte((d & 1 ? bf16_hi(v) : bf16_lo(v)) * vinv));
            else reinterpret_cast<uint16_t *>(vp)[at] = static_cast<uint16_t>(d & 1 ? v >> 16 : v);
        }
        return;
    }
    // sixteen places of two components each
    const int c0 = F8 && vfac != 1.f ? 0 : lo >> 4, nc = ((hi + 15) >> 4) - c0;
    const FastDiv by_nc = a.by_chunks[nc];
    for (int e = tid; e < nc * (D / 2); e += kCacheThreads) {
        const int d2 = quot(by_nc, e), p0 = (c0 + (e - d2 * nc)) * 16;
        char *dst = vp + ((static_cast<int64_t>(2 * d2) << a.c.log_page) + p0) * EB;
        const int64_t next = static_cast<int64_t>(EB) << a.c.log_page;     // bytes to the next component
        const bool whole = p0 >= lo && p0 + 16 <= hi;
        uint32_t v[16];                                     // two components of each place
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int p = p0 + i;
            v[i] = whole || (p >= lo && p < hi) ? s_v[(p - lo) * VW + d2] : 0u;
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            u32x4 w[EB];
            if (!whole) {
#pragma unroll
                for (int i = 0; i < EB; ++i) w[i] = reinterpret_cast<const u32x4 *>(dst + y * next)[i];
            }
            if constexpr (F8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float f[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) f[q] = (y ? bf16_hi(v[4 * i + q]) : bf16_lo(v[4 * i + q])) * vinv;
                    const uint32_t fresh = f8_quad(f[0], f[1], f[2], f[3]);
                    if (whole) {
                        w[0][i] = fresh;
                    } else {
                        uint32_t is_new = 0, is_old = 0;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int p = p0 + 4 * i + q;
                            is_new |= p >= lo && p < hi ? 0xffu << (8 * q) : 0u;
                            is_old |= p < lo ? 0xffu << (8 * q) : 0u;
                        }
                        uint32_t kept = w[0][i];
                        if (vfac != 1.f) kept = (f8_rescaled(kept, vfac) & is_old) | (kept & ~is_old);
                        w[0][i] = (fresh & is_new) | (kept & ~is_new);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t fresh = y ? (v[2 * i] >> 16) | (v[2 * i + 1] & 0xffff0000u)
                                             : (v[2 * i] & 0xffffu) | (v[2 * i + 1] << 16);
                    if (whole) {
                        w[i / 4][i % 4] = fresh;
                    } else {
                        const int p = p0 + 2 * i;
                        const uint32_t is_new = (p >= lo && p < hi ? 0xffffu : 0u) | (p + 1 >= lo && p + 1 < hi ? 0xffff0000u : 0u);
                        w[i / 4][i % 4] = (fresh & is_new) | (w[i / 4][i % 4] & ~is_new);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < EB; ++i) reinterpret_cast<u32x4 *>(dst + y * next)[i] = w[i];
        }
    }
}

// One workgroup per (sequence, head, keys or values) moves the path's places.  A path's ids increase, so
// a place comes from its own position or a later one: the places of as many pages as kMaxPage
// places hold are taken to LDS before any is written, and what later places come from has not been
// written then.  The table's entries and the scales of all pages that hold nodes are read first, at once.
template <int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void k_cache_keep(KeepArgs a) {
    constexpr int EB = F8 ? 1 : 2;
    constexpr int RS = D * EB + 16;
    constexpr int kPages = kMaxSeqRows / 16 + 1;            // that N nodes can lie in
    __shared__ __attribute__((aligned(16))) char s_x[kMaxPage * RS];
    __shared__ int s_path[kMaxSeqRows];
    __shared__ int s_page[kPages];                          // or -1
    __shared__ float s_scale[kPages];                       // present ones
    __shared__ int s_fresh[kPages], s_moves[kPages];        // a page's new scale (its bits), whether a node moves in
    __shared__ int s_len;
    const int tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    const uint32_t bh = blockIdx.x >> 1;
    const int b = quot(a.by_heads, bh), h = bh - b * a.by_heads.d;
    const int log_page = a.c.log_page, P = 1 << log_page;
    char *mem = values ? a.c.v : a.c.k;
    float *scales = values ? a.c.v_scale : a.c.k_scale;
    int node = -1;
    if (tid < a.N) node = a.path[static_cast<int64_t>(b) * a.N + tid];
    const int64_t ctx = max(a.ctx_len[b], 0);
    const int64_t j0 = ctx >> log_page;                     // first page
    const int first = static_cast<int>(ctx & (P - 1));      // its places before the nodes hold earlier positions
    if (tid < kPages) {
        int64_t id = -1;
        if (j0 + tid < a.c.max_pages)
            id = page_or_none(a.c, a.c.table[static_cast<int64_t>(b) * a.c.max_pages + j0 + tid]);
        s_page[tid] = static_cast<int>(id);
        s_scale[tid] = F8 && id >= 0 ? power_of(scales[id * a.c.H + h]) : 1.f;
        s_fresh[tid] = 0;
        s_moves[tid] = 0;
    }
    if (tid == 0) s_len = a.N;
    __syncthreads();
    if (tid < a.N) {
        s_path[tid] = node;
        if (node < 0 || node >= a.N) atomicMin(&s_len, tid);
    }
    __syncthreads();
    const int len = s_len;
    // position i of the nodes: page (first + i) >> log_page of those in LDS, place (first + i) & (P - 1)
    const int64_t head_bytes = static_cast<int64_t>(D * EB) << log_page;
    auto block_at = [&](int page) { return mem + (static_cast<int64_t>(s_page[page]) * a.c.H + h) * head_bytes; };
    if (tid < len) {
        const int to = (first + tid) >> log_page, from = (first + node) >> log_page;
        if (s_page[to] >= 0 && s_page[from] >= 0) {
            atomicMax(&s_fresh[to], __float_as_int(s_scale[from]));
            if (node != tid) s_moves[to] = 1;
        }
    }
    __syncthreads();
    if (tid == 0 && first > 0) s_fresh[0] = max(s_fresh[0], __float_as_int(s_scale[0]));
    // whether position i is written, and from where
    auto moved = [&](int i) {
        const int to = (first + i) >> log_page;
        return s_moves[to] && s_page[(first + s_path[i]) >> log_page] >= 0;
    };
    for (int i0 = 0; i0 < len;) {
        // whole pages of places, as many as are held
        int T = P - ((first + i0) & (P - 1));
        while (i0 + T < len && T + P <= kMaxPage) T += P;
        T = min(T, len - i0);
        __syncthreads();                                    // the places held before are used up
        if (values) {
            for (int e = tid; e < T * D; e += kCacheThreads) {
                const int t = e / D, d = e % D;
                if (!moved(i0 + t)) continue;
                const int at = first + s_path[i0 + t];
                const char *src = block_at(at >> log_page) + ((static_cast<int64_t>(d) << log_page) + (at & (P - 1))) * EB;
                if constexpr (F8) s_x[t * RS + d] = *src;
                else *reinterpret_cast<uint16_t *>(s_x + t * RS + d * 2) = *reinterpret_cast<const uint16_t *>(src);
            }
        } else {
            constexpr int CPR = D * EB / 16;
            for (int e = tid; e < T * CPR; e += kCacheThreads) {
                const int t = e / CPR, c = e % CPR;
                if (!moved(i0 + t)) continue;
                const int at = first + s_path[i0 + t];
                *reinterpret_cast<u32x4 *>(s_x + t * RS + c * 16) =
                    *reinterpret_cast<const u32x4 *>(block_at(at >> log_page) + static_cast<int64_t>(at & (P - 1)) * (D * EB) + c * 16);
            }
        }
        __syncthreads();
        auto factor = [&](int i) {                          // from the source's scale to the new one
            return s_scale[(first + s_path[i]) >> log_page] / __int_as_float(s_fresh[(first + i) >> log_page]);
        };
        if (values) {
            for (int e = tid; e < T * D; e += kCacheThreads) {
                const int d = e / T, t = e - d * T, at = first + i0 + t;
                if (!moved(i0 + t)) continue;
                char *dst = block_at(at >> log_page) + ((static_cast<int64_t>(d) << log_page) + (at & (P - 1))) * EB;
                if constexpr (F8) *dst = static_cast<char>(f8_byte(f8_value(static_cast<uint8_t>(s_x[t * RS + d])) * factor(i0 + t)));
                else *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(s_x + t * RS + d * 2);
            }
        } else {
            constexpr int CPR = D * EB / 16;
            for (int e = tid; e < T * CPR; e += kCacheThreads) {
                const int t = e / CPR, c = e % CPR, at = first + i0 + t;
                if (!moved(i0 + t)) continue;
                u32x4 w = *reinterpret_cast<const u32x4 *>(s_x + t * RS + c * 16);
                if constexpr (F8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = f8_rescaled(w[i], factor(i0 + t));
                }
                *reinterpret_cast<u32x4 *>(block_at(at >> log_page) + static_cast<int64_t>(at & (P - 1)) * (D * EB) + c * 16) = w;
            }
        }
        i0 += T;
    }
    if constexpr (F8) {
        if (tid < kPages && s_moves[tid]) scales[static_cast<int64_t>(s_page[tid]) * a.c.H + h] = __int_as_float(s_fresh[tid]);
        if (s_moves[0] && first > 0 && __int_as_float(s_fresh[0]) != s_scale[0]) {
            const float f = s_scale[0] / __int_as_float(s_fresh[0]);
            char *page = block_at(0);
            for (int e = tid; e < first * D; e += kCacheThreads) {
                char *p = page + (values ? (static_cast<int64_t>(e / first) << log_page) + e % first : e);
                *p = static_cast<char>(f8_byte(f8_value(static_cast<uint8_t>(*p)) * f));
            }
        }
    }
}

template <int D, bool F8> void run_append(const AppendArgs &a, unsigned grid, size_t lds, hipStream_t s) {
    if (a.interleaved) hipLaunchKernelGGL((k_cache_append<D, F8, 1>), dim3(grid), dim3(kCacheThreads), lds, s, a);
    else hipLaunchKernelGGL((k_cache_append<D, F8, 0>), dim3(grid), dim3(kCacheThreads), lds, s, a);
}

}  // namespace

hipError_t launch_cache_append(AppendArgs a, hipStream_t s) {
    const int64_t pages = pages_touched(a.n, a.c.log_page);
    const int64_t page_wgs = a.B * pages * a.c.H;
    const int64_t query_wgs = a.q ? (static_cast<int64_t>(a.B) * a.n + kQueryTokens - 1) / kQueryTokens : 0;
    a.page_wgs = static_cast<uint32_t>(page_wgs);
    a.by_pages = fast_div(static_cast<uint32_t>(pages));
    a.by_heads = fast_div(a.c.H);
    a.by_n = fast_div(a.n);
    for (int i = 1; i <= kMaxPage / 16; ++i) a.by_chunks[i] = fast_div(i);
    const unsigned grid = static_cast<unsigned>(page_wgs + query_wgs);
    // the value rows of as many tokens as a page can get, or the queries' cos and sin
    const int tokens = a.n < (1 << a.c.log_page) ? a.n : 1 << a.c.log_page;
    const size_t rows = static_cast<size_t>(tokens) * (a.c.D / 2 + 1) * 4;
    const size_t lds = std::max(rows, a.q ? static_cast<size_t>(kQueryTokens) * (a.c.D / 2) * 8 : 0);
    if (a.c.D == 128) a.c.f8 ? run_append<128, true>(a, grid, lds, s) : run_append<128, false>(a, grid, lds, s);
    else a.c.f8 ? run_append<64, true>(a, grid, lds, s) : run_append<64, false>(a, grid, lds, s);
    return hipGetLastError();
}

hipError_t launch_cache_keep(KeepArgs a, hipStream_t s) {
    a.by_heads = fast_div(a.c.H);
    const dim3 grid(static_cast<unsigned>(a.B * a.c.H * 2)), block(kCacheThreads);
    if (a.c.D == 128) {
        if (a.c.f8) hipLaunchKernelGGL((k_cache_keep<128, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((k_cache_keep<128, false>), grid, block, 0, s, a);
    } else {
        if (a.c.f8) hipLaunchKernelGGL((k_cache_keep<64, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((k_cache_keep<64, false>), grid, block, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace cospec
