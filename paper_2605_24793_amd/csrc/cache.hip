// Writing the paged key/value cache: appending new positions (keys rotated to their place,
// values transposed into the pages' layout, queries rotated beside them) and keeping the
// accepted path of a token tree.
//
// 8-bit pages hold e4m3 values with one power-of-two scale per page and head.  A floating type
// loses nothing to a scale's mantissa, and with powers of two a page whose scale grows keeps its
// earlier values' bits (only the exponents move; what becomes subnormal is rounded once more).
#include "paged.h"

namespace cospec {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float floatx2;

constexpr int kCacheThreads = 256;
constexpr int kMaxPage = 128;
constexpr int kQueryTokens = 8;       // tokens of a query workgroup
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

// cos and sin of position * inv_freq: reduced to a fraction of a turn in double precision
// (far positions then lose nothing; the rest, sine and cosine of a fraction, is fp32).
__device__ inline float2 turn(int64_t position, float inv_freq) {
    const double turns = static_cast<double>(position) * static_cast<double>(inv_freq) * 0.15915494309189535;
    float s, c;
    sincospif(2.f * static_cast<float>(turns - rint(turns)), &s, &c);
    return make_float2(c, s);
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

// The unit's sixteen values (run a, then run b), rotated by cs = {cos, sin} of its pairs.
__device__ inline void load_unit(const char *row, const Unit &u, int interleaved, const float2 *cs, float *x) {
    unpack8(*reinterpret_cast<const u32x4 *>(row + u.a * 2), x);
    unpack8(*reinterpret_cast<const u32x4 *>(row + u.b * 2), x + 8);
    if (u.pair < 0) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 t = cs[u.pair + i];
        const int p1 = interleaved ? 2 * i : i, p2 = interleaved ? 2 * i + 1 : i + 8;
        const float x1 = x[p1], x2 = x[p2];
        x[p1] = x1 * t.x - x2 * t.y;
        x[p2] = x2 * t.x + x1 * t.y;
    }
}

template <int INTERLEAVED>
__device__ inline void load_rotated(const char *row, const Unit &u, const float2 *cs, float *x) {
    load_unit(row, u, INTERLEAVED, cs, x);
}

__device__ inline void store_bf16(char *row, const Unit &u, const float *x) {
    *reinterpret_cast<u32x4 *>(row + u.a * 2) =
        u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
    *reinterpret_cast<u32x4 *>(row + u.b * 2) =
        u32x4{bf16_pair(x[8], x[9]), bf16_pair(x[10], x[11]), bf16_pair(x[12], x[13]), bf16_pair(x[14], x[15])};
}

// One workgroup per (sequence, page it touches, head) writes the page's new keys and values,
// or, from workgroup page_wgs on, rotates the queries of kQueryTokens tokens.
//
// Keys: a thread holds its units' rotated values in registers while the workgroup finds their
// largest, so they are read once and rounded once.  Values: staged in LDS as rows, read as
// columns, since a page holds them transposed; a thread writes sixteen places of a
// component at a time (16 or 32 bytes), merged with what the page holds where only some of them are new.
template <int D, bool F8, int INTERLEAVED>
__global__ __launch_bounds__(kCacheThreads) void k_cache_append(AppendArgs a) {
    constexpr int UPT = D / 16;                             // units of a token's head
    constexpr int MAXU = kMaxPage * UPT / kCacheThreads;    // units of a thread
    constexpr int EB = F8 ? 1 : 2;
    constexpr int VS = D * 2 + 4;                           // bytes of a staged value row: odd in words
    __shared__ __attribute__((aligned(16))) char s_v[kMaxPage * VS];
    __shared__ float2 s_cs[kMaxPage * D / 2];
    __shared__ float s_max[2][kCacheThreads / 64];
    const int tid = threadIdx.x, pairs = a.rot / 2;

    if (blockIdx.x >= a.page_wgs) {                         // queries
        const int64_t t0 = static_cast<int64_t>(blockIdx.x - a.page_wgs) * kQueryTokens;
        const int T = static_cast<int>(min(static_cast<int64_t>(kQueryTokens), static_cast<int64_t>(a.B) * a.n - t0));
        for (int e = tid; e < T * pairs; e += kCacheThreads) {
            const int t = e / pairs, i = e - t * pairs;
            const int64_t tok = t0 + t;
            const int b = quot(a.by_n, static_cast<uint32_t>(tok));
            const int64_t pos = a.positions ? a.positions[tok] : a.start[b] + (tok - static_cast<int64_t>(b) * a.n);
            s_cs[e] = turn(pos, a.inv_freq[i]);
        }
        __syncthreads();
        const int per = a.Hq * UPT;
        for (int e = tid; e < T * per; e += kCacheThreads) {
            const int t = e / per, hu = e - t * per;
            const int h = hu / UPT;
            const Unit u = unit_of(hu % UPT, a.rot, INTERLEAVED);
            float x[16];
            load_rotated<INTERLEAVED>(a.q + ((t0 + t) * a.ld_q + h * D) * 2, u, s_cs + t * pairs, x);
            store_bf16(a.q_out + ((t0 + t) * a.Hq + h) * D * 2, u, x);
        }
        return;
    }

    const int P = 1 << a.c.log_page;
    const uint32_t bj = quot(a.by_heads, blockIdx.x);
    const int h = blockIdx.x - bj * a.by_heads.d;
    const int b = quot(a.by_pages, bj);
    const int64_t start = a.start[b];
    const int64_t cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const int64_t j = (max(start, static_cast<int64_t>(0)) >> a.c.log_page) + (bj - b * a.by_pages.d);
    // places [lo, hi) of the page are new; token of place s: base + s
    const int64_t base = j * P - start;
    const int lo = static_cast<int>(max(static_cast<int64_t>(0), -base));
    const int hi = static_cast<int>(min(static_cast<int64_t>(P), cnt - base));
    if (lo >= hi || j >= a.c.max_pages) return;
    const int64_t pid = page_or_none(a.c, a.c.table[static_cast<int64_t>(b) * a.c.max_pages + j]);
    if (pid < 0) return;
    const int T = hi - lo;
    const int64_t tok0 = static_cast<int64_t>(b) * a.n + base + lo;    // row of the first new token
    const int64_t blk = pid * a.c.H + h;

    for (int e = tid; e < T * pairs; e += kCacheThreads) {
        const int t = e / pairs, i = e - t * pairs;
        const int64_t pos = a.positions ? a.positions[tok0 + t] : start + base + lo + t;
        s_cs[e] = turn(pos, a.inv_freq[i]);
    }
    // values: rows to LDS
    float vmax = 0.f;
    for (int e = tid; e < T * (D / 8); e += kCacheThreads) {
        const int t = e / (D / 8), c8 = e % (D / 8);
        const u32x4 w = *reinterpret_cast<const u32x4 *>(a.v + ((tok0 + t) * a.ld_v + h * D + c8 * 8) * 2);
        uint32_t *dst = reinterpret_cast<uint32_t *>(s_v + t * VS + c8 * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            dst[i] = w[i];
            vmax = fmaxf(vmax, fmaxf(finite_abs(bf16_lo(w[i])), finite_abs(bf16_hi(w[i]))));
        }
    }
    __syncthreads();
    // keys: rotated in registers
    float x[MAXU][16], kmax = 0.f;
#pragma unroll
    for (int m = 0; m < MAXU; ++m) {
        const int e = m * kCacheThreads + tid;
        if (e >= T * UPT) break;
        const int t = e / UPT;
        load_rotated<INTERLEAVED>(a.k + ((tok0 + t) * a.ld_k + h * D) * 2, unit_of(e % UPT, a.rot, INTERLEAVED),
                                  s_cs + t * pairs, x[m]);
#pragma unroll
        for (int i = 0; i < 16; ++i) kmax = fmaxf(kmax, finite_abs(x[m][i]));
    }
    // scales: lo places of the page hold earlier positions of this sequence
    float kinv = 1.f, vinv = 1.f, kfac = 1.f, vfac = 1.f;
    if constexpr (F8) {
        float ks = scale_for(max_group(kmax, s_max[0])), vs = scale_for(max_group(vmax, s_max[1]));
        if (lo > 0) {
            const float ko = power_of(a.c.k_scale[blk]), vo = power_of(a.c.v_scale[blk]);
            ks = fmaxf(ks, ko);
            vs = fmaxf(vs, vo);
            kfac = ko / ks;
            vfac = vo / vs;
        }
        kinv = 1.f / ks;
        vinv = 1.f / vs;
        __syncthreads();                                    // every thread has read the present scales
        if (tid == 0) {
            a.c.k_scale[blk] = ks;
            a.c.v_scale[blk] = vs;
        }
    }
    char *kp = a.c.k + (blk << a.c.log_page) * (D * EB);
#pragma unroll
    for (int m = 0; m < MAXU; ++m) {
        const int e = m * kCacheThreads + tid;
        if (e >= T * UPT) break;
        const Unit u = unit_of(e % UPT, a.rot, INTERLEAVED);
        char *row = kp + static_cast<int64_t>(lo + e / UPT) * (D * EB);
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
    // values: sixteen places of a component each
    char *vp = a.c.v + (blk << a.c.log_page) * (D * EB);
    const int c0 = F8 && vfac != 1.f ? 0 : lo >> 4, nc = ((hi + 15) >> 4) - c0;
    for (int e = tid; e < nc * D; e += kCacheThreads) {
        const int d = e % D, p0 = (c0 + e / D) * 16;
        char *dst = vp + ((static_cast<int64_t>(d) << a.c.log_page) + p0) * EB;
        const bool whole = p0 >= lo && p0 + 16 <= hi;
        u32x4 w[EB];
        if (!whole) {
#pragma unroll
            for (int i = 0; i < EB; ++i) w[i] = reinterpret_cast<const u32x4 *>(dst)[i];
        }
        if constexpr (F8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t q = 0;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int p = p0 + 4 * i + s;
                    uint32_t byte;
                    if (p >= lo && p < hi) {
                        const uint32_t v = *reinterpret_cast<const uint16_t *>(s_v + (p - lo) * VS + d * 2);
                        byte = f8_byte(__uint_as_float(v << 16) * vinv);
                    } else {
                        byte = (w[0][i] >> (8 * s)) & 0xffu;
                        if (p < lo && vfac != 1.f) byte = f8_byte(f8_value(byte) * vfac);
                    }
                    q |= byte << (8 * s);
                }
                w[0][i] = q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t q = 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int p = p0 + 2 * i + s;
                    const uint32_t v = p >= lo && p < hi ? *reinterpret_cast<const uint16_t *>(s_v + (p - lo) * VS + d * 2)
                                                         : (w[i / 4][i % 4] >> (16 * s)) & 0xffffu;
                    q |= v << (16 * s);
                }
                w[i / 4][i % 4] = q;
            }
        }
#pragma unroll
        for (int i = 0; i < EB; ++i) reinterpret_cast<u32x4 *>(dst)[i] = w[i];
    }
}

// One workgroup per (sequence, head, keys or values) moves the path's places, page by page of
// where they go.  A path's ids increase, so a page's places come from that page or later
// ones: all of them are taken to LDS before any is written, and no later page has been
// written yet.
template <int D, bool F8>
__global__ __launch_bounds__(kCacheThreads) void k_cache_keep(KeepArgs a) {
    constexpr int EB = F8 ? 1 : 2;
    constexpr int RS = D * EB + 4;
    __shared__ __attribute__((aligned(16))) char s_x[kMaxPage * RS];
    __shared__ int s_path[kMaxSeqRows];
    __shared__ float s_scale[kMaxPage];                     // of each place's source; < 0: no source
    __shared__ float s_max[kCacheThreads / 64];
    __shared__ int s_len, s_moves;
    const int tid = threadIdx.x;
    const bool values = blockIdx.x & 1;
    const uint32_t bh = blockIdx.x >> 1;
    const int b = quot(a.by_heads, bh), h = bh - b * a.by_heads.d;
    const int P = 1 << a.c.log_page;
    if (tid == 0) s_len = a.N;
    __syncthreads();
    for (int i = tid; i < a.N; i += kCacheThreads) {
        const int node = a.path[static_cast<int64_t>(b) * a.N + i];
        s_path[i] = node;
        if (node < 0 || node >= a.N) atomicMin(&s_len, i);
    }
    __syncthreads();
    const int len = s_len;
    const int64_t ctx = max(a.ctx_len[b], 0);
    const int32_t *table = a.c.table + static_cast<int64_t>(b) * a.c.max_pages;
    char *mem = values ? a.c.v : a.c.k;
    float *scales = values ? a.c.v_scale : a.c.k_scale;
    // byte of component d of place p: keys are rows of a place, values of a component
    const int64_t step_p = values ? EB : D * EB, step_d = values ? static_cast<int64_t>(P) * EB : EB;

    for (int i0 = 0; i0 < len;) {
        const int64_t j = (ctx + i0) >> a.c.log_page;
        const int held = static_cast<int>((ctx + i0) & (P - 1));   // places before: of this sequence, in the first page
        const int T = min(len - i0, P - held);
        if (j >= a.c.max_pages) break;
        const int64_t pid = page_or_none(a.c, table[j]);
        const int64_t blk = pid * a.c.H + h;
        __syncthreads();                                    // the last page's staged places are used up
        if (tid == 0) s_moves = 0;
        __syncthreads();
        for (int t = tid; t < T; t += kCacheThreads) {
            const int64_t from = ctx + s_path[i0 + t];
            float sc = -1.f;
            if (pid >= 0 && (from >> a.c.log_page) < a.c.max_pages) {
                const int64_t sp = page_or_none(a.c, table[from >> a.c.log_page]);
                if (sp >= 0) {
                    sc = F8 ? power_of(scales[sp * a.c.H + h]) : 1.f;
                    if (s_path[i0 + t] != i0 + t) s_moves = 1;
                }
            }
            s_scale[t] = sc;
        }
        __syncthreads();
        if (!s_moves) {                                     // every node of this page stands in its place
            i0 += T;
            continue;
        }
        for (int e = tid; e < T * D; e += kCacheThreads) {
            const int t = values ? e % T : e / D, d = values ? e / T : e % D;
            if (s_scale[t] < 0.f) continue;
            const int64_t from = ctx + s_path[i0 + t];
            const int64_t sblk = static_cast<int64_t>(table[from >> a.c.log_page]) * a.c.H + h;
            const char *src = mem + (sblk << a.c.log_page) * (D * EB) + (from & (P - 1)) * step_p + d * step_d;
            if constexpr (F8) s_x[t * RS + d] = *src;
            else *reinterpret_cast<uint16_t *>(s_x + t * RS + d * 2) = *reinterpret_cast<const uint16_t *>(src);
        }
        float fresh = 1.f, fac = 1.f;
        if constexpr (F8) {
            float m = 0.f;
            for (int t = tid; t < T; t += kCacheThreads) m = fmaxf(m, s_scale[t]);
            fresh = max_group(m, s_max);
            const float old = power_of(scales[blk]);
            if (held > 0) {
                fresh = fmaxf(fresh, old);
                fac = old / fresh;
            }
        }
        __syncthreads();                                    // staged, and the present scales are read
        if (F8 && tid == 0) scales[blk] = fresh;
        char *page = mem + (blk << a.c.log_page) * (D * EB);
        for (int e = tid; e < T * D; e += kCacheThreads) {
            const int t = values ? e % T : e / D, d = values ? e / T : e % D;
            if (s_scale[t] < 0.f) continue;
            char *dst = page + (held + t) * step_p + d * step_d;
            if constexpr (F8) {
                const uint32_t byte = static_cast<uint8_t>(s_x[t * RS + d]);
                *dst = static_cast<char>(s_scale[t] == fresh ? byte : f8_byte(f8_value(byte) * (s_scale[t] / fresh)));
            } else {
                *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(s_x + t * RS + d * 2);
            }
        }
        if (F8 && fac != 1.f) {
            for (int e = tid; e < held * D; e += kCacheThreads) {
                char *p = page + (values ? e % held : e / D) * step_p + (values ? e / held : e % D) * step_d;
                *p = static_cast<char>(f8_byte(f8_value(static_cast<uint8_t>(*p)) * fac));
            }
        }
        i0 += T;
    }
}

template <int D, bool F8> void run_append(const AppendArgs &a, unsigned grid, hipStream_t s) {
    if (a.interleaved) hipLaunchKernelGGL((k_cache_append<D, F8, 1>), dim3(grid), dim3(kCacheThreads), 0, s, a);
    else hipLaunchKernelGGL((k_cache_append<D, F8, 0>), dim3(grid), dim3(kCacheThreads), 0, s, a);
}

}  // namespace

hipError_t launch_cache_append(AppendArgs a, hipStream_t s) {
    // pages a sequence's n positions can touch, wherever they start
    const int64_t pages = ((static_cast<int64_t>(a.n) + (1 << a.c.log_page) - 2) >> a.c.log_page) + 1;
    const int64_t page_wgs = a.B * pages * a.c.H;
    const int64_t query_wgs = a.q ? (static_cast<int64_t>(a.B) * a.n + kQueryTokens - 1) / kQueryTokens : 0;
    a.page_wgs = static_cast<uint32_t>(page_wgs);
    a.by_pages = fast_div(static_cast<uint32_t>(pages));
    a.by_heads = fast_div(a.c.H);
    a.by_n = fast_div(a.n);
    const unsigned grid = static_cast<unsigned>(page_wgs + query_wgs);
    if (a.c.D == 128) a.c.f8 ? run_append<128, true>(a, grid, s) : run_append<128, false>(a, grid, s);
    else a.c.f8 ? run_append<64, true>(a, grid, s) : run_append<64, false>(a, grid, s);
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
