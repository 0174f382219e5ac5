// What the attentions over pages share (paged_attention.hip, latent_attention.hip): vectors and
// matrix products, loads from global memory into LDS, which keys a query sees, how keys are cut into
// pieces, which workgroup takes what.
#pragma once

#include "paged.h"

namespace cospec {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef __attribute__((ext_vector_type(16))) float floatx16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;             // of a workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kSegment = 252;         // pages looked up at a time: with one more, at most one a thread; whole turns
constexpr int kStep = 64;             // keys of a wave's turn, at most
constexpr int64_t kMaxPieces = 64;    // of a group's keys (the join weighs them in one wave)
constexpr int64_t kCus = 256;         // compute units of an MI355X
constexpr uint32_t kNone = 0x80000000u;   // marks a table entry that names no page
constexpr float kLog2eP = 1.4426950408889634f;
constexpr float kLazyRescale = 8.0f;  // log2 units a block's max may exceed the running max by

__device__ inline uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

__device__ inline floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

__device__ inline floatx16 mfma32(u32x4 a, u32x4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// max over the four lanes that share a query column (l % 16)
__device__ inline float max_rows(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// Eight e4m3 bytes (two words) times a power of two, as four words of two bf16.
__device__ inline u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}

// The highest bit of every element of four bytes that is not finite (e4m3: `carry` 0x01010101; with
// 0x08080808 also those over 240).
template <bool F8> __device__ inline uint32_t not_finite(uint32_t x, uint32_t carry) {
    return F8 ? ((x & 0x7f7f7f7fu) + carry) & 0x80808080u : ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// A value that is the same in every lane, for the scalar registers.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A load through the scalar cache, of what no kernel writes while this one runs.
typedef __attribute__((address_space(4))) const int const_int;
__device__ inline int scalar_load(const int32_t *p) { return *(const_int *)reinterpret_cast<uintptr_t>(p); }

// What the queries of sequence b see.  Hybrid: position p < lc sees [0, p], lc <= p < end sees
// [0, end).  Tree: node r sees [0, lc) and its ancestors among lc .. end - 1.
struct Seq {
    int lc, end;
    int64_t qs;
};

__device__ inline Seq sequence_of(const PagedArgs &a, int b) {
    const int64_t room = static_cast<int64_t>(a.c.max_pages) << a.c.log_page;
    const int64_t lc = max(scalar_load(a.ctx_len + b), 0);
    const int64_t more = a.parent ? a.n_q : 2 * static_cast<int64_t>(a.K) + 3;
    const int end = static_cast<int>(min(lc + more, room));
    return Seq{static_cast<int>(min(lc, static_cast<int64_t>(end))), end, a.parent ? lc : static_cast<int64_t>(scalar_load(a.q_start + b))};
}

// Keys [0, kend) that the rows [q0, q1) of a group see, and how they are cut.
struct Cut {
    int kend, chunk;
    int pieces;                // at least 1
};

__device__ inline Cut cut_of(const PagedArgs &a, const Seq &s, int q0, int q1) {
    const int64_t p_lo = s.qs + quot(a.by_grp, q0), p_hi = s.qs + quot(a.by_grp, q1 - 1);
    int kend = s.end;
    if (p_lo >= s.end) kend = 0;                            // all padding: no key
    else if (!a.parent && p_hi < s.lc) kend = max(static_cast<int>(p_hi) + 1, 0);
    const Pieces p = pieces_of(kend, quot(a.by_splits, kend + a.splits - 1), kStep, a.min_piece);
    return Cut{kend, p.chunk, p.count};
}

// Keys [0, result) of a piece's [.., kend) are seen by every row of [q0, q1) that sees any.
__device__ inline int seen_by_all(const PagedArgs &a, const Seq &s, int q0, int kend) {
    if (a.parent) return min(s.lc, kend);
    const int64_t p = max(s.qs + quot(a.by_grp, q0), static_cast<int64_t>(0));
    return p >= s.lc ? kend : min(static_cast<int>(p) + 1, kend);
}

// The sixteen bits from bit `at` (may be negative) of a set of 256.
__device__ inline uint32_t window16(const uint32_t *set, int at) {
    if (at <= -16 || at >= 256) return 0;
    if (at < 0) return (set[0] << -at) & 0xffffu;
    const int w = at >> 5;
    const uint64_t two = set[w] | static_cast<uint64_t>(w < 7 ? set[w + 1] : 0u) << 32;
    return static_cast<uint32_t>(two >> (at & 31)) & 0xffffu;
}

// 16 bytes per lane from global memory into LDS at byte lds + 16 * lane, lds the same in every
// lane.  Written as assembly, so that the compiler, which knows nothing of these loads, places no
// wait for them before LDS reads; the kernel's own waits order them.  ONCE: read once, not to be kept in
// the caches.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool ONCE> __device__ inline void load_lds16(const char *src, uint32_t lds) {
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(lds), "v"(src) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

// 16 (or 4) bytes per lane from base + off[i] + 1024 i, off an offset of the lane's own, into LDS at byte lds + 1024 i +
// 16 * lane (4 * lane).  A wave that loads while another one multiplies gets its vector instructions into the few
// cycles between products: so the lanes' offsets are made once, and a turn's addresses are scalar.  (See load_lds16.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int N> __device__ inline void load_lds_rows(const char *base, const uint32_t *off, uint32_t lds) {
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1"
                     : : "s"(lds), "s"(base), "v"(off[0]) : "memory", "m0");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024"
                     : : "s"(lds), "s"(base), "v"(off[0]), "v"(off[1]) : "memory", "m0");
    else {
        static_assert(N % 4 == 0);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1\n\tglobal_load_lds_dwordx4 %3, %1 offset:1024\n\t"
                     "global_load_lds_dwordx4 %4, %1 offset:%6\n\tglobal_load_lds_dwordx4 %5, %1 offset:%7"
                     : : "s"(lds), "s"(base), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "i"(2 * 1024), "i"(3 * 1024)
                     : "memory", "m0");
        if constexpr (N > 4) load_lds_rows<N - 4>(base + 4096, off + 4, lds + 4096);
    }
}

__device__ inline void load_lds4(const char *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %2, %1" : : "s"(lds), "s"(base), "v"(off) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until at most N vector-memory operations of this wave are outstanding.
template <int N> __device__ inline void wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// Waits for this wave's LDS reads.
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

typedef __attribute__((address_space(3))) const char lds_cchar;

// Workgroup barrier that does not wait for the loads still in flight (as the fence of
// __syncthreads would); the compiler may not move memory accesses across it.
__device__ inline void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Ancestors of every node, as sets of 256 bits in LDS, by all threads: each round joins the set
// of the node `up`, twice as far up as the round before.  Up to 64 nodes are one wave's, which needs no barriers
// (16 trees of 60 nodes over bf16 latents 137.2 us with them, 135.0 without; one tree over bf16 pages 12.5 and 11.6).
__device__ inline void find_ancestors(const PagedArgs &a, int b, uint32_t (*s_anc)[8], int *s_up) {
    const int tid = threadIdx.x;
    const int n = a.n_q;
    int up = -1;
    if (n <= 64) {
        if (tid < 64) {
            if (tid < n) {
                const int p = a.parent[static_cast<int64_t>(b) * n + tid];
                up = p >= 0 && p < tid ? p : -1;
            }
            uint32_t set[2] = {tid < 32 ? 1u << tid : 0u, tid < 32 ? 0u : 1u << (tid - 32)};
            for (int far = 1; far < n; far *= 2) {
                const int from = up >= 0 ? up : tid;
                const uint32_t lo = __shfl(set[0], from), hi = __shfl(set[1], from);
                const int next_up = __shfl(up, from);
                set[0] |= lo;                               // (a node's own set where there is none above)
                set[1] |= hi;
                up = next_up;
            }
            if (tid < n) {
#pragma unroll
                for (int w = 0; w < 8; ++w) s_anc[tid][w] = w < 2 ? set[w] : 0u;
            }
        }
        __syncthreads();
        return;
    }
    if (tid < n) {
        const int p = a.parent[static_cast<int64_t>(b) * n + tid];
        up = p >= 0 && p < tid ? p : -1;
#pragma unroll
        for (int w = 0; w < 8; ++w) s_anc[tid][w] = w == tid >> 5 ? 1u << (tid & 31) : 0u;
        s_up[tid] = up;
    }
    for (int far = 1; far < n; far *= 2) {
        __syncthreads();
        uint32_t set[8];
        int next_up = -1;
#pragma unroll
        for (int w = 0; w < 8; ++w) set[w] = up >= 0 ? s_anc[up][w] : 0u;
        if (up >= 0) next_up = s_up[up];
        __syncthreads();
        if (tid < n) {
#pragma unroll
            for (int w = 0; w < 8; ++w) s_anc[tid][w] |= set[w];
            s_up[tid] = up = next_up;
        }
    }
    __syncthreads();
}

// Which rows, keys and group a workgroup takes.  Workgroups are dealt to the XCDs round-robin: those
// that read the same keys (the row blocks of a piece of a group) follow each other on one XCD,
// whose L2 then serves all but the first; the last rows, which see the most keys, come first.
struct Place {
    int b, h, block, piece;
};

__device__ inline Place place_of(const PagedArgs &a) {
    const uint32_t slot = blockIdx.x / kXcds;
    const uint32_t round = quot(a.by_blocks, slot);
    const int block = a.by_blocks.d - 1 - (slot - round * a.by_blocks.d);
    const uint32_t unit = round * kXcds + blockIdx.x % kXcds;
    const uint32_t bh = quot(a.by_splits, unit);
    const int b = quot(a.by_heads, bh);
    return Place{b, static_cast<int>(bh - b * a.by_heads.d), block, static_cast<int>(unit - bh * a.by_splits.d)};
}

// This thread's entry of sequence b's table, from entry `first` on (clamped to the table).
__device__ inline uint32_t table_entry(const PagedArgs &a, int b, int first) {
    const int at = min(first + static_cast<int>(threadIdx.x), a.c.max_pages - 1);
    return a.c.table[static_cast<int64_t>(b) * a.c.max_pages + at];
}

__device__ inline uint32_t lds_address(const void *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_cchar *)p));
}

// The 32 bits from bit `at` (may be negative) of a set of 256.
__device__ inline uint32_t window32(const uint32_t *set, int at) { return window16(set, at) | window16(set, at + 16) << 16; }

// Bits 0 .. n - 1, n clamped to 0 .. 32.
__device__ inline uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

}  // namespace
}  // namespace cospec
