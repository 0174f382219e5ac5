// Attention over the paged key/value cache: the arbitrator's hybrid attention and the
// attention of token-tree nodes, for any number of queries per sequence.
//
// Online softmax: with scores s_j = scale * q . k_j, a running max m and the sums
// l = sum_j 2^(s_j log2 e - m), o = sum_j 2^(s_j log2 e - m) v_j, one pass over the keys gives
// o / l; raising m multiplies both sums by 2^(m_old - m_new), and sums over disjoint keys are
// joined the same way.
//
// Work split: the query rows (position x head) that share a key/value head of a sequence form
// a group.  A workgroup takes rows of a group; with up to 48 of them (96 of many groups' workgroups) its waves
// take turns at the group's keys (k_paged_attention): a wave's keys and values of a turn go from the
// pages into LDS of its own with loads that pass no register, each lane's operands where the
// lane reads them back, so that the wave has its next turn under way without a barrier, and the
// waves' sums are joined at the end.  With more rows the waves take rows of their own and share
// the keys (k_paged_attention_wide).  Few groups are cut over their keys into pieces,
// by each sequence's own length, which a second kernel joins.
//
// S^T = K Q^T (v_mfma_f32_16x16x32_bf16): lane l holds query column l % 16, so the softmax of a
// query stays in four lanes.  Which key stands in which row of a product is free: row i of
// tile t is key 16 (i / 4) + 4 t + i % 4 of the 64, so that lane l's scores are the 16 keys
// 16 (l / 16) + 4 t + r, in order.  These are also, as they stand, a lane's share of the
// second product's operand P^T, and the values it needs for them are 16 keys in a row: with
// values kept [d][place] they are 16 (e4m3) or 32 (bf16) contiguous bytes.
//
// The weights are rounded to bf16 for that product, and l sums the rounded ones (in fp32, by the matrix cores: 16 additions
// a query and turn less on the vector unit), so that what rounding does to all of them alike leaves the
// quotient.  Relative error against 64 bits: 0.0017 to 0.0020, with weights and sums of 32 bits 0.0017, which is the
// output's own rounding.
//
// e4m3: v_cvt_scalef32_pk_bf16_fp8 widens two elements and applies the page's power of two;
// e4m3 has fewer bits than bf16, so nothing is rounded, and one conversion serves all rows.
#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace cospec {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;             // of a workgroup
constexpr int kThreads = 64 * kWaves;
constexpr int kSegment = 252;         // pages looked up at a time: with one more, at most one a thread; whole turns
constexpr int kStep = 64;             // keys of a wave's turn, at most
// 16-row tiles of a workgroup, at most: what the registers hold of queries, scores and sums
constexpr int kMaxRowTiles = 3;
// Keys of a piece, at least.  One token at 15000 positions: pieces of 256 17.6 us, 512 15.0, 1024 17.0; with many rows
// (196 of a group at 4687) 25.7, 24.3 and 33.5.
constexpr int kMinPiece = 512;
constexpr int kMinPieceWide = 256;
constexpr int64_t kMaxPieces = 64;    // of a group's keys (the join weighs them in one wave)
constexpr float kLog2eP = 1.4426950408889634f;
constexpr float kLazyRescale = 8.0f;  // log2 units a block's max may exceed the running max by

__device__ inline uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

__device__ inline floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
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

// Values that are not finite, among keys that some rows see and others do not.  A weight of zero would not keep them
// from the others: they are made zero, and the weights of the rows that do see such a key NaN.
// not_finite: the highest bit of every such element of four bytes (e4m3: `carry` is 0x01010101, or at the scale 2^120
// 0x08080808, as more than 240 times that is not finite in bf16); emptied: the four bytes without these elements;
// element_bits: one bit per element of not_finite's.
template <bool F8> __device__ inline uint32_t not_finite(uint32_t x, uint32_t carry) {
    return F8 ? ((x & 0x7f7f7f7fu) + carry) & 0x80808080u : ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

__device__ inline uint32_t carry_of(float scale) { return scale < 1.329227995784916e36f ? 0x01010101u : 0x08080808u; }

template <bool F8> __device__ inline uint32_t emptied(uint32_t x, uint32_t top) {
    return x & ~(top | (top - (top >> (F8 ? 7 : 15))));
}

template <bool F8> __device__ inline uint32_t element_bits(uint32_t top) {
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < (F8 ? 4 : 2); ++e) bits |= (top >> (F8 ? 8 * e + 7 : 16 * e + 15) & 1u) << e;
    return bits;
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
// of the node `up`, twice as far up as the round before.
__device__ inline void find_ancestors(const PagedArgs &a, int b, uint32_t (*s_anc)[8], int *s_up) {
    const int tid = threadIdx.x;
    const int n = a.n_q;
    int up = -1;
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

// What a workgroup keeps in LDS of each page of its keys, up to kThreads of them at a time, one looked
// up by each thread: {page * heads + head, with kNone for a page that is none (it is read as page
// 0, and not used); the upper halves of the scales of keys and of values (e4m3)}.
typedef uint2 PageEntry;
constexpr uint32_t kNone = 0x80000000u;

// (2^120 is the largest scale that an append writes; no scale, of a page in use or not, makes a zero anything else)
__device__ inline uint32_t pack_scales(float k, float v) {
    const uint32_t most = 0x7b800000u;
    return min(__float_as_uint(k) & 0x7f800000u, most) | min(__float_as_uint(v) & 0x7f800000u, most) >> 16;
}
__device__ inline float key_scale(PageEntry e) { return __uint_as_float(e.y & 0xffff0000u); }
__device__ inline float value_scale(PageEntry e) { return __uint_as_float(e.y << 16); }

// This thread's entry of sequence b's table, from entry `first` on (clamped to the table).
__device__ inline uint32_t table_entry(const PagedArgs &a, int b, int first) {
    const int at = min(first + static_cast<int>(threadIdx.x), a.c.max_pages - 1);
    return a.c.table[static_cast<int64_t>(b) * a.c.max_pages + at];
}

// RW waves of the four share the keys, each with RT row tiles of its own; the 4 / RW sets of them
// take turns at the keys.
//
// A round of 64 sequences at 1536 to 2065 positions, 32/8 heads, D = 128, e4m3 (68 rows a group, 255 MB, 32 GFLOP):
// 61.5 us, 4.1 TB/s.  Its vector and matrix instructions share one issue port and fill 70% of the
// time a wave is there; a workgroup starts to work some 8 us after its launch, and
// sequences of different lengths leave 1.4 waves per SIMD on average.  Measured on the way: keys and values in
// registers with no LDS 114, through LDS (a wave's next turn in flight without a register) 87, 48 rows a wave
// and no branch to choose a page 77, two waves sharing keys 69, the weights' sum by the matrix
// cores and raised priority there 65.7, no turns for a tile without rows 61.5.  64 single tokens at about 3600 positions (471 MB): 80 us, 5.9 TB/s.
// A fifth row tile per wave spills (190 us); a wave alone on its SIMD, whatever its rows, is slower than two.
template <int D, bool F8, int RT, int RW, bool ONCE = false>
__global__ __launch_bounds__(kThreads, 2) void k_paged_attention(PagedArgs a) {
    constexpr int DS = D / 32;                              // k-steps of the first product
    constexpr int DT = D / 16;                              // d tiles of the second
    constexpr int EB = F8 ? 1 : 2;
    constexpr int KS = D * EB > 128 ? 32 : 64;              // keys of a turn: 16 KB with their values
    constexpr int NT = KS / 16, NU = KS / 32;               // key tiles, and k-steps of the second product
    constexpr int HT = RT > 2 ? 1 : NT / 2, HD = RT > 2 ? 1 : DT / 2;   // key and component tiles whose operands are held at a time
    constexpr int GK = KS / 4;                              // keys of a lane group
    constexpr int KC = D * EB / 64;                         // 16-byte pieces of a lane's key
    constexpr int VC = GK * EB / 16;                        // ... and of its values of a component
    constexpr int NK = NT * KC, NV = DT * VC;               // loads of a turn's keys, and values
    constexpr int KW = kWaves / RW;                         // sets of waves
    constexpr int NS = RW;                                  // turns of a set that are in LDS at a time
    constexpr int kValuesAt = NK * 1024, kStage = (NK + NV) * 1024;
    constexpr int OS = D + 4;                               // floats of a staged row of sums
    constexpr int kLds = kWaves * (kStage > 16 * OS * 4 ? kStage : 16 * OS * 4);
    static_assert(NK % RW == 0 && NV % RW == 0 && KW * NS == kWaves, "turns");
    __shared__ __attribute__((aligned(16))) char s_ring[kLds];
    __shared__ float2 s_ml[kWaves][16 * RT];
    __shared__ PageEntry s_page[kThreads];
    __shared__ uint32_t s_anc[kMaxSeqRows][8];
    __shared__ int s_up[kMaxSeqRows];
    // where waves share turns: {first key of a turn, which of a lane group's keys in it have values that are not finite},
    // as the wave found them before it made these zero
    __shared__ uint2 s_bad[kWaves][4];

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int rw = wave % RW, kw = wave / RW;
    const int g = lane >> 4, l16 = lane & 15, kg = l16 >> 2;
    const int grp = a.by_grp.d, rows = a.n_q * grp;
    const Place w_ = place_of(a);
    const int b = w_.b, h = w_.h, piece = w_.piece;
    if (b >= a.B) return;
    const int q0 = w_.block * (16 * RT * RW), q1 = min(q0 + 16 * RT * RW, rows);
    // what the loads below need is known: they go out before the sequence's length is
    uint32_t id = a.splits == 1 ? table_entry(a, b, 0) : 0u;
    // This lane's query of every row tile.  Keys are taken by a k-step as they lie in memory:
    // bf16 key bytes 64 c + 16 g .. + 15, k-step c; e4m3 the same bytes, k-steps 2c and 2c + 1.
    u32x4 qf[RT][DS];
    int node[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int qi = min(q0 + (rw * RT + rt) * 16 + l16, q1 - 1);
        node[rt] = quot(a.by_grp, qi);
        const int hq = h * grp + (qi - node[rt] * grp);
        const char *qrow = static_cast<const char *>(a.q) + ((static_cast<int64_t>(b) * a.n_q + node[rt]) * a.Hq + hq) * D * 2;
#pragma unroll
        for (int c = 0; c < DS; ++c) {
            const int d = F8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
            qf[rt][c] = *reinterpret_cast<const u32x4 *>(qrow + d * 2);
        }
    }
    const Seq s = sequence_of(a, b);
    const Cut cut = cut_of(a, s, q0, q1);
    if (piece >= cut.pieces) return;
    const int kbeg = piece * cut.chunk, kend = min(kbeg + cut.chunk, cut.kend);

    // The pages of up to kSegment pages' keys are looked up at a time, by all threads, into LDS.
    const int P1 = (1 << a.c.log_page) - 1;
    const char *const set_lds = s_ring + kw * NS * kStage;
    const uint32_t ring = uniform(static_cast<int>(reinterpret_cast<uintptr_t>((lds_cchar *)set_lds)));
    int first_page = 0, last_page = 0;                      // of those in LDS
    uint32_t scales = 0;
    auto look_up = [&](int from, int to, uint32_t entry) {  // of keys [from, to), this thread's table entry given
        first_page = from >> a.c.log_page;
        last_page = (to - 1) >> a.c.log_page;
        const bool in = tid <= last_page - first_page, none = entry >= static_cast<uint32_t>(a.c.n_pages);
        const uint32_t at = (none ? 0 : entry) * a.c.H + h;
        if (in) s_page[tid].x = at | (none ? kNone : 0u);
        if (F8 && in) scales = pack_scales(a.c.k_scale[at], a.c.v_scale[at]);
    };
    // This lane's key rows of a turn are among the keys GK kg .. GK kg + GK - 1, its values those of
    // the keys GK g ..: each within one page.
    // (keys past the last one are looked for in the last page, and not used)
    auto page_of = [&](int key) { return s_page[min(key >> a.c.log_page, last_page) - first_page]; };
    // this wave's share of a turn's keys and values, into LDS at `at`
    auto load_keys = [&](int k0, uint32_t at) {
        const int key = k0 + kg * GK;
        const PageEntry page = page_of(key);
        const char *base = a.c.k + ((static_cast<int64_t>(page.x & ~kNone) << a.c.log_page) + (key & P1) + (l16 & 3)) * (D * EB) + g * 16;
#pragma unroll
        for (int i = 0; i < NK / RW; ++i) {
            const int e = rw * (NK / RW) + i;
            load_lds16<ONCE>(base + (e / KC) * 4 * (D * EB) + (e % KC) * 64, at + e * 1024);
        }
    };
    const int64_t v_tile = (static_cast<int64_t>(16) << a.c.log_page) * EB;
    auto load_values = [&](int k0, uint32_t at) {
        const int key = k0 + g * GK;
        const PageEntry page = page_of(key);
        const char *base = a.c.v + (((static_cast<int64_t>(page.x & ~kNone) * D + l16) << a.c.log_page) + (key & P1)) * EB;
#pragma unroll
        for (int i = 0; i < NV / RW; ++i) {
            const int e = rw * (NV / RW) + i;
            load_lds16<ONCE>(base + (e / VC) * v_tile + (e % VC) * 16, at + kValuesAt + e * 1024);
        }
    };
    constexpr int kTurn = KW * KS;                          // keys of all sets' turns
    const int segment = kSegment << a.c.log_page;
    if (a.parent) find_ancestors(a, b, s_anc, s_up);

    // Scores are taken as |scale| (+-q) . k, so that the largest product is the largest score.
    int vis[RT];                                            // keys [0, vis) are seen
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int64_t p = s.qs + node[rt];
        const bool live = q0 + (rw * RT + rt) * 16 + l16 < q1 && p >= 0 && p < s.end;
        vis[rt] = !live ? 0 : a.parent ? s.lc : p >= s.lc ? s.end : static_cast<int>(p) + 1;
        if (!live) node[rt] = -1;
#pragma unroll
        for (int c = 0; c < DS; ++c)
#pragma unroll
            for (int w = 0; w < 4; ++w) qf[rt][c][w] = live ? qf[rt][c][w] ^ flip : 0u;
    }
    const int clear = seen_by_all(a, s, q0, kend);          // turns that end here or before mask nothing

    floatx4 o[RT][DT];
    float m[RT];
    floatx4 ol[RT];                                         // sums of the weights alone, rows all alike
    const u32x4 ones{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        ol[rt] = floatx4{0.f, 0.f, 0.f, 0.f};
        m[rt] = -INFINITY;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[rt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float sc = fmaxf(fabsf(a.scale) * kLog2eP, 1.17549435e-38f);
    if (RW > 1 && tid < kWaves * 4) s_bad[tid / 4][tid % 4].x = kNone;       // no key
    auto attend = [&](auto tiles) {                         // the wave's first R row tiles
        constexpr int R = decltype(tiles)::value;
        for (int seg = kbeg; seg < kend; seg += segment) {
            const int seg_end = min(seg + segment, kend);
            if (seg > kbeg || a.splits > 1) id = table_entry(a, b, seg >> a.c.log_page);
            if (seg > kbeg) __syncthreads();                    // the pages of the segment before are used up
            look_up(seg, seg_end, id);
            lds_barrier();
            const int k_first = seg + kw * KS;
            const int turns = k_first < seg_end ? (seg_end - k_first + kTurn - 1) / kTurn : 0;
            const int all_turns = (seg_end - seg + kTurn - 1) / kTurn;   // of the set that has most
            if (turns > 0) {                                    // a set is one turn ahead in its loads
                load_keys(k_first, ring);
                load_values(k_first, ring);
            }
            if (F8 && tid <= last_page - first_page) s_page[tid].y = scales;
            lds_barrier();
            for (int j = 0; j < (RW > 1 ? all_turns : turns); ++j) {
                const int k0 = k_first + j * kTurn;
                const bool more = j + 1 < turns;
                const uint32_t at = RW > 1 ? (j % NS) * kStage : 0;
                const u32x4 *keys = reinterpret_cast<const u32x4 *>(set_lds + at) + lane;
                u32x4 *values = reinterpret_cast<u32x4 *>(s_ring + kw * NS * kStage + at + kValuesAt) + lane;
                if constexpr (RW > 1) {
                    wait_vm<0>();                               // this wave's loads of the turn
                    lds_barrier();                              // ... and the others'; the turn before is used up
                    if (more) {
                        const uint32_t to = ring + ((j + 1) % NS) * kStage;
                        load_keys(k0 + kTurn, to);
                        load_values(k0 + kTurn, to);
                    }
                    if (j >= turns) continue;                   // wave-uniform; another set has one more
                }
                const float ksc = key_scale(page_of(k0 + kg * GK));
                const PageEntry page_v = page_of(k0 + g * GK);
                const float vsc = value_scale(page_v);
                const bool none = page_v.x >= kNone;
                // wave-uniform: a key that some query does not see, or that does not exist
                const bool masked = k0 + KS > clear || __ballot(none) != 0;
                // S^T of the turn
                floatx4 st[R][NT];
                if (RW == 1) wait_vm<NV>();                         // its keys have landed
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int th = 0; th < NT; th += HT) {
                    u32x4 kf[HT][DS];
#pragma unroll
                    for (int t = 0; t < HT; ++t) {
                        u32x4 raw[KC];
#pragma unroll
                        for (int c = 0; c < KC; ++c) raw[c] = keys[((th + t) * KC + c) * 64];
#pragma unroll
                        for (int c = 0; c < DS; ++c) {
                            if constexpr (F8) kf[t][c] = widen(raw[c / 2][2 * (c % 2)], raw[c / 2][2 * (c % 2) + 1], ksc);
                            else kf[t][c] = raw[c];
                        }
                    }
#pragma unroll
                    for (int rt = 0; rt < R; ++rt)
#pragma unroll
                        for (int t = 0; t < HT; ++t) st[rt][th + t] = floatx4{0.f, 0.f, 0.f, 0.f};
                    // products that follow each other are of different sums
#pragma unroll
                    for (int i = 0; i < DS * R; ++i) {
                        const int c = RT > 2 ? i / R : i % DS, rt = RT > 2 ? i % R : i / DS;
#pragma unroll
                        for (int t = 0; t < HT; ++t) st[rt][th + t] = mfma(kf[t][c], qf[rt][c], st[rt][th + t]);
                    }
                }
                __builtin_amdgcn_s_setprio(0);
                if constexpr (RW == 1) {
                    wait_lds();
                    if (more) load_keys(k0 + kTurn, ring);
                }
                if (masked) {
                    const int kb = k0 + g * GK;                     // this lane's first key
                    const int real = none ? 0 : min(max(kend - kb, 0), GK);
#pragma unroll
                    for (int rt = 0; rt < R; ++rt) {
                        const int top = min(max(vis[rt] - kb, 0), real);
                        uint32_t see = (1u << top) - 1u;
                        if (a.parent && node[rt] >= 0) see |= window16(s_anc[node[rt]], kb - s.lc) & ((1u << real) - 1u);
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (!(see >> (4 * t + r) & 1)) st[rt][t][r] = -INFINITY;
                    }
                }
                float bm[R];
                bool raise = false;
#pragma unroll
                for (int rt = 0; rt < R; ++rt) {
                    bm[rt] = -INFINITY;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) bm[rt] = fmaxf(bm[rt], st[rt][t][r]);
                    bm[rt] = max_rows(bm[rt]) * sc;
                    raise |= bm[rt] > m[rt] + kLazyRescale;         // always when m is still -inf
                }
                if (__builtin_expect(__ballot(raise) != 0, 0)) {
#pragma unroll
                    for (int rt = 0; rt < R; ++rt) {
                        const bool up = bm[rt] > m[rt] + kLazyRescale;
                        const float alpha = up ? __builtin_amdgcn_exp2f(m[rt] - bm[rt]) : 1.f;   // 0 from -inf
                        if (up) m[rt] = bm[rt];
                        ol[rt] *= alpha;
#pragma unroll
                        for (int t = 0; t < DT; ++t) o[rt][t] *= alpha;
                    }
                }
                // O^T += V^T P^T
                if constexpr (RW == 1) {
                    if (more) wait_vm<NK>();
                    else wait_vm<0>();
                }
                if (masked) {
                    // places that hold no key of the sequence may hold anything: a weight of zero does not make
                    // a NaN harmless
                    const int real = none ? 0 : min(max(kend - (k0 + g * GK), 0), GK);
                    constexpr int EW = 4 / EB;                      // elements of a word
                    if (__ballot(real < GK) != 0) {
#pragma unroll
                        for (int c = 0; c < VC; ++c) {
                            u32x4 keep;
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                const int in = real - (c * 4 + w) * EW;
                                keep[w] = in >= EW ? 0xffffffffu : in > 0 ? (1u << (in * 8 * EB)) - 1u : 0u;
                            }
                            // (waves that share the turn store the same)
#pragma unroll
                            for (int t = 0; t < DT; ++t) values[(t * VC + c) * 64] &= keep;
                        }
                    }
                    if (k0 + KS > clear && clear < kend) {          // some rows do not see all of them
                        uint32_t top[VC * 4] = {}, any = 0;
                        const uint32_t carry = carry_of(vsc);
#pragma unroll
                        for (int c = 0; c < VC; ++c)
#pragma unroll
                            for (int t = 0; t < DT; ++t) {
                                const u32x4 x = values[(t * VC + c) * 64];
#pragma unroll
                                for (int w = 0; w < 4; ++w) top[c * 4 + w] |= not_finite<F8>(x[w], carry);
                            }
#pragma unroll
                        for (int i = 0; i < VC * 4; ++i) any |= top[i];
                        // Where another wave has made zero what this one would have found, it has said so before: it is
                        // asked after the search.  (The values are read again for the products: kept in registers
                        // they spill.)
                        wait_lds();
                        uint32_t others = 0;
                        int here = g;
                        if constexpr (RW > 1) {
                            asm volatile("" : "+v"(here));          // (its address in no register between turns)
                            static_assert(RW == 2, "one other wave");
                            const uint2 other = s_bad[wave ^ 1][here];
                            others = other.x == static_cast<uint32_t>(k0) ? other.y : 0u;
                        }
                        if (__builtin_expect(__ballot((any | others) != 0) != 0, 0)) {
                            uint32_t bad = others;                  // keys of this lane group
#pragma unroll
                            for (int i = 0; i < VC * 4; ++i) bad |= element_bits<F8>(top[i]) << (i * EW);
#pragma unroll
                            for (int off = 1; off < 16; off <<= 1) bad |= __shfl_xor(bad, off);
                            if constexpr (RW > 1) {
                                s_bad[wave][here] = make_uint2(k0, bad);
                                wait_lds();
                            }
#pragma unroll
                            for (int c = 0; c < VC; ++c)
#pragma unroll
                                for (int t = 0; t < DT; ++t) {
                                    u32x4 x = values[(t * VC + c) * 64];
#pragma unroll
                                    for (int w = 0; w < 4; ++w) x[w] = emptied<F8>(x[w], not_finite<F8>(x[w], carry));
                                    values[(t * VC + c) * 64] = x;
                                }
#pragma unroll
                            for (int rt = 0; rt < R; ++rt)
#pragma unroll
                                for (int t = 0; t < NT; ++t)
#pragma unroll
                                    for (int r = 0; r < 4; ++r)
                                        if ((bad >> (4 * t + r) & 1u) && st[rt][t][r] != -INFINITY) st[rt][t][r] = NAN;
                        }
                    }
                }
                u32x4 pb[R][NU];
#pragma unroll
                for (int rt = 0; rt < R; ++rt) {
                    // a query that has seen nothing yet keeps m = -inf and adds nothing
                    const float mm = m[rt] == -INFINITY ? INFINITY : m[rt];
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        float p[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(st[rt][2 * u + i / 4][i % 4], sc, -mm));
                        pb[rt][u] = u32x4{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3]), bf16_pair(p[4], p[5]), bf16_pair(p[6], p[7])};
                    }
                }
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int rt = 0; rt < R; ++rt) ol[rt] = mfma(ones, pb[rt][u], ol[rt]);
#pragma unroll
                for (int th = 0; th < DT; th += HD) {
                    u32x4 vf[HD][NU];
#pragma unroll
                    for (int t = 0; t < HD; ++t) {
                        u32x4 raw[VC];
#pragma unroll
                        for (int c = 0; c < VC; ++c) raw[c] = values[((th + t) * VC + c) * 64];
#pragma unroll
                        for (int u = 0; u < NU; ++u) {
                            if constexpr (F8) vf[t][u] = widen(raw[0][2 * u], raw[0][2 * u + 1], vsc);
                            else vf[t][u] = raw[u];
                        }
                    }
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int rt = 0; rt < R; ++rt)
#pragma unroll
                            for (int t = 0; t < HD; ++t) o[rt][th + t] = mfma(vf[t][u], pb[rt][u], o[rt][th + t]);
                }
                __builtin_amdgcn_s_setprio(0);
                if constexpr (RW == 1) {
                    wait_lds();
                    if (more) load_values(k0 + kTurn, ring);
                }
            }
        }
    };
    // Of up to 80 rows the second wave's third tile has none: left out, 68 rows take 61.5 us, with it 65.7.  (Of
    // workgroups whose waves take the same rows it is not worth the code: 30.3 and 30.4 for two long sequences.)
    bool all_tiles = true;
    if constexpr (RW > 1 && RT > 2) {
        all_tiles = q0 + (rw * RT + RT - 1) * 16 < q1;
        if (!all_tiles) attend(std::integral_constant<int, RT - 1>{});
    }
    if (all_tiles) attend(std::integral_constant<int, RT>{});

    // join the sets
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const bool live = node[rt] >= 0;                    // else unmasked turns gave it some weights
        if (!live) m[rt] = -INFINITY;
        if (g == 0) s_ml[wave][rt * 16 + l16] = make_float2(m[rt], live ? ol[rt][0] : 0.f);
    }
    const bool whole = cut.pieces == 1;
    const int64_t rows_all = static_cast<int64_t>(a.B) * a.n_q * a.Hq;
    constexpr int TPR = kThreads / (16 * RW);               // threads of a row, four components each at a time
    float *s_o = reinterpret_cast<float *>(s_ring);         // [kWaves][16][OS]
    __syncthreads();                                    // every wave is done with its turns
    const int row = tid / TPR % 16, rw_ = tid / TPR / 16, d0 = tid % TPR * 4;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW; ++w) M = fmaxf(M, s_ml[w * RW + rw][rt * 16 + l16].x);
        const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - M);
#pragma unroll
        for (int t = 0; t < DT; ++t)
            *reinterpret_cast<floatx4 *>(s_o + (wave * 16 + l16) * OS + t * 16 + g * 4) = node[rt] >= 0 ? o[rt][t] * f : floatx4{0.f, 0.f, 0.f, 0.f};
        __syncthreads();
        const int qi = q0 + (rw_ * RT + rt) * 16 + row;
        float RM = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) RM = fmaxf(RM, s_ml[w * RW + rw_][rt * 16 + row].x);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            const float2 ml = s_ml[w * RW + rw_][rt * 16 + row];
            L += ml.x == -INFINITY ? 0.f : ml.y * __builtin_amdgcn_exp2f(ml.x - RM);
        }
        const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;       // NaN stays
        const int r = quot(a.by_grp, min(qi, q1 - 1));
        const int64_t R = (static_cast<int64_t>(b) * a.n_q + r) * a.Hq + h * grp + (min(qi, q1 - 1) - r * grp);
#pragma unroll
        for (int i = 0; i < D; i += 4 * TPR) {
            floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < KW; ++w)
                x += *reinterpret_cast<const floatx4 *>(s_o + ((w * RW + rw_) * 16 + row) * OS + d0 + i);
            if (qi < q1) {
                if (whole)
                    *reinterpret_cast<u32x2 *>(static_cast<char *>(a.out) + (R * D + d0 + i) * 2) =
                        u32x2{bf16_pair(x[0] * inv, x[1] * inv), bf16_pair(x[2] * inv, x[3] * inv)};
                else
                    *reinterpret_cast<floatx4 *>(a.part_o + (piece * rows_all + R) * D + d0 + i) = x;
            }
        }
        if (!whole && qi < q1 && d0 == 0) a.part_ml[piece * rows_all + R] = make_float2(RM, L);
        __syncthreads();                                // the staged sums are read
    }
}

// ---------------------------------------------------------------- many query rows

typedef __attribute__((ext_vector_type(16))) float floatx16;

constexpr int kWideRows = 32 * kWaves;

__device__ inline floatx16 mfma32(u32x4 a, u32x4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// The same attention where a group has many query rows.  There the vector unit bounds it: every
// instruction, a matrix one too, takes it for 4 to 5 cycles.  So each wave takes 32 rows with 32 x 32
// products (half as many instructions), and the workgroup widens a turn's 64 keys and values once,
// for its four waves: each takes a quarter through its registers into LDS, in the order of the
// products' operands, while the turn before is worked on.
//
// Whole inputs of 4 x 1820 to 2063 positions, 32/8 heads, D = 128, e4m3 (121 GFLOP): 161 us, 753 TFLOP/s; trees of
// 60 nodes after 64 contexts of 1536 to 2048 (113 GFLOP) 164 us.  No pipe is full: matrix instructions take 36% of
// the time, vector ones 31% on the same port, the LDS reads of the operands (1 KB a product of 32 cycles) 43%; the
// waits between them bound it.  Without those reads the same code takes 116 to 125 us, without staging 124 to 132,
// without the products 139 to 145, without the exponentials 150.  Measured and not
// taken: 16 x 16 products 163 to 175, each wave widening for itself 170, products and weights interleaved by
// scheduling groups 157 to 168, 32-key turns with three workgroups a CU 165 to 178, 64 rows a wave spills.
//
// S^T = K Q^T: row p of key tile kt is its key 16 (p / 4 % 2) + 4 (p / 8) + p % 4, so that lane half
// gh's sixteen scores are those of the keys 16 gh + 0 .. 15 in order, P^T's operand as they stand.
//
// (three workgroups of e4m3, d = 64 fit on a CU: 95.4 us for such inputs, 101 with the registers of two)
template <int D, bool F8>
__global__ __launch_bounds__(kThreads, D == 64 && F8 ? 3 : 2) void k_paged_attention_wide(PagedArgs a) {
    constexpr int KS = 64, KT = KS / 32;                    // keys of a turn, and tiles of them
    constexpr int DS = D / 16, DT = D / 32;                 // k-steps of the first product, component tiles
    constexpr int EB = F8 ? 1 : 2;
    constexpr int CPR = D * EB / 16;                        // 16-byte pieces of a key row
    constexpr int LK = KS * CPR / kThreads;                 // of a turn's keys, of one thread
    constexpr int CPD = KS * EB / 16, LV = D * CPD / kThreads;  // of a component's values, and of one thread
    constexpr int kValuesAt = KS * D * 2, kStage = 2 * kValuesAt;
    __shared__ __attribute__((aligned(16))) char s_stage[2][kStage];
    __shared__ PageEntry s_page[kThreads];
    __shared__ uint32_t s_anc[kMaxSeqRows][8];
    __shared__ int s_up[kMaxSeqRows];
    __shared__ int s_met;                                   // values that are not finite, among keys that not all rows see
    // with care: the 64 keys of a turn that have such values; of the turn that is worked on, of the one that is staged
    // meanwhile, and of the one before, which are cleared
    __shared__ uint32_t s_bad[3][2];

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int gh = lane >> 5, l32 = lane & 31;
    const int grp = a.by_grp.d, rows = a.n_q * grp;
    const Place w = place_of(a);
    if (w.b >= a.B) return;
    const int b = w.b, h = w.h;
    const int q0 = w.block * kWideRows, q1 = min(q0 + kWideRows, rows);
    // what the loads below need is known: they go out before the sequence's length is
    uint32_t id = a.splits == 1 ? table_entry(a, b, 0) : 0u;
    const int qi = q0 + wave * 32 + l32;                    // this lane's query
    const bool valid = qi < q1;
    const int r = quot(a.by_grp, min(qi, q1 - 1));
    const int64_t R = (static_cast<int64_t>(b) * a.n_q + r) * a.Hq + h * grp + (min(qi, q1 - 1) - r * grp);
    u32x4 qf[DS];
#pragma unroll
    for (int c = 0; c < DS; ++c)
        qf[c] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + (R * D + c * 16 + gh * 8) * 2);
    const Seq s = sequence_of(a, b);
    const Cut cut = cut_of(a, s, q0, q1);
    if (w.piece >= cut.pieces) return;
    const int kbeg = w.piece * cut.chunk, kend = min(kbeg + cut.chunk, cut.kend);
    const int all_see = seen_by_all(a, s, q0, kend);        // keys below are seen by every row that sees any

    const int P1 = (1 << a.c.log_page) - 1;
    int first_page = 0, last_page = 0;                      // of those in LDS
    bool any_none = false;                                  // among them
    auto page_of = [&](int key) { return s_page[min(key >> a.c.log_page, last_page) - first_page]; };
    // piece i of this thread: of key row key_at(i) the bytes 16 key_piece(i) .. + 15, and of component
    // comp_at(i) the keys 16 / EB * comp_piece(i) ..; sixteen lanes side by side take sixteen rows, of keys
    // those that are side by side in the products' order too (consecutive ones meet in LDS banks: 4 x 2048
    // positions of bf16, d = 64, 67.2 us; now 61.2; the same in e4m3, d = 128, 160 and 160)
    auto key_at = [&](int i) {
        const int t = (wave * LK + i) / (CPR / 4);
        return (t >> 1) * 32 + ((lane >> 2) & 1) * 16 + (t & 1) * 8 + ((lane >> 3) & 1) * 4 + (lane & 3);
    };
    auto key_piece = [&](int i) { return (wave * LK + i) % (CPR / 4) * 4 + (lane >> 4); };
    auto comp_at = [&](int i) { return ((wave * LV + i) / (CPD / 4)) * 16 + (lane & 15); };
    auto comp_piece = [&](int i) { return (wave * LV + i) % (CPD / 4) * 4 + (lane >> 4); };
    u32x4 kr[LK], vr[LV];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LK; ++i) {
            const int key = k0 + key_at(i);
            const int64_t at = page_of(key).x & ~kNone;
            kr[i] = *reinterpret_cast<const u32x4 *>(
                a.c.k + ((at << a.c.log_page) + (key & P1)) * (D * EB) + key_piece(i) * 16);
        }
#pragma unroll
        for (int i = 0; i < LV; ++i) {
            const int key = k0 + comp_piece(i) * (16 / EB);
            const int64_t at = page_of(key).x & ~kNone;
            vr[i] = *reinterpret_cast<const u32x4 *>(
                a.c.v + (((at * D + comp_at(i)) << a.c.log_page) + (key & P1)) * EB);
        }
    };
    // widened into LDS; values of places that hold no key of the sequence become zeros (such places
    // may hold anything, and a weight of zero does not make a NaN harmless)
    // (inlined by request: a call puts what it captures on the stack)
    auto stage = [&](int k0, char *to, uint32_t *bad, auto with_care) __attribute__((always_inline)) {
        constexpr bool CARE = decltype(with_care)::value;
#pragma unroll
        for (int i = 0; i < LK; ++i) {
            const int key = key_at(i), k32 = key & 31;
            const int p = ((k32 >> 2) & 3) * 8 + (k32 >> 4) * 4 + (k32 & 3);
            char *tile = to + (key >> 5) * (DS * 1024) + p * 16;
            if constexpr (F8) {
                const float scale = key_scale(page_of(k0 + key));
                *reinterpret_cast<u32x4 *>(tile + key_piece(i) * 1024) = widen(kr[i][0], kr[i][1], scale);
                *reinterpret_cast<u32x4 *>(tile + key_piece(i) * 1024 + 512) = widen(kr[i][2], kr[i][3], scale);
            } else {
                *reinterpret_cast<u32x4 *>(tile + (key_piece(i) >> 1) * 1024 + (key_piece(i) & 1) * 512) = kr[i];
            }
        }
        const bool some_see = k0 + KS > all_see && all_see < kend, special = some_see || k0 + KS > kend || any_none;
#pragma unroll
        for (int i = 0; i < LV; ++i) {
            const int at = comp_piece(i) * (16 / EB);        // first of the piece's keys
            const PageEntry page = page_of(k0 + at);
            const float scale = value_scale(page);
            constexpr int EW = 4 / EB;
            if (special) {
                const int real = page.x >= kNone ? 0 : min(max(kend - (k0 + at), 0), 16 / EB);
                uint32_t met = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int in = real - x * EW;
                    vr[i][x] &= in >= EW ? 0xffffffffu : in > 0 ? (1u << (in * 8 * EB)) - 1u : 0u;
                    if (!CARE && some_see) {
                        const uint32_t top = not_finite<F8>(vr[i][x], 0x01010101u);
                        met |= top;
                        vr[i][x] = emptied<F8>(vr[i][x], top);
                    }
                }
                if (!CARE && met != 0) s_met = 1;
            }
            if constexpr (CARE) {
                uint32_t keys = 0;                           // of the piece's, from its first one on
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t top = not_finite<F8>(vr[i][x], carry_of(scale));
                    keys |= element_bits<F8>(top) << (x * EW);
                    vr[i][x] = emptied<F8>(vr[i][x], top);
                }
                if (keys) atomicOr(&bad[at >> 5], keys << (at & 31));
            }
            const int d = comp_at(i);
            // operand of component tile d / 32, key tile at / 32, k-step v: keys 16 gh + 8 v ..
            char *tile = to + kValuesAt + (((d >> 5) * KT + (at >> 5)) * 2) * 1024 + ((d & 31) + 32 * ((at >> 4) & 1)) * 16;
            if constexpr (F8) {
                *reinterpret_cast<u32x4 *>(tile) = widen(vr[i][0], vr[i][1], scale);
                *reinterpret_cast<u32x4 *>(tile + 1024) = widen(vr[i][2], vr[i][3], scale);
            } else {
                *reinterpret_cast<u32x4 *>(tile + ((at >> 3) & 1) * 1024) = vr[i];
            }
        }
    };
    const int segment = kSegment << a.c.log_page;
    auto look_up = [&](int from, int to, uint32_t entry) {  // of keys [from, to), this thread's table entry given
        first_page = from >> a.c.log_page;
        last_page = (to - 1) >> a.c.log_page;
        const bool in = tid <= last_page - first_page, none = entry >= static_cast<uint32_t>(a.c.n_pages);
        const uint32_t at = (none ? 0 : entry) * a.c.H + h;
        if (in) s_page[tid].x = at | (none ? kNone : 0u);
        uint32_t scales = 0;
        if (F8 && in) scales = pack_scales(a.c.k_scale[at], a.c.v_scale[at]);
        any_none = __syncthreads_or(in && none);
        load(from);
        if (F8 && in) {
            s_page[tid].y = scales;
            if (carry_of(__uint_as_float(scales << 16)) != 0x01010101u) s_met = 1;   // values over 240 need care
        }
        __syncthreads();
    };
    if (a.parent) find_ancestors(a, b, s_anc, s_up);

    // scores are taken as |scale| (+-q) . k, so that the largest product is the largest score
    const int64_t p_q = s.qs + r;
    const bool live = valid && p_q >= 0 && p_q < s.end;
    const int vis = !live ? 0 : a.parent ? s.lc : p_q >= s.lc ? s.end : static_cast<int>(p_q) + 1;   // keys [0, vis) are seen
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int c = 0; c < DS; ++c)
#pragma unroll
        for (int x = 0; x < 4; ++x) qf[c][x] = live ? qf[c][x] ^ flip : 0u;
    int vis_min = live ? vis : INT32_MAX;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) vis_min = min(vis_min, __shfl_xor(vis_min, off));
    const int clear = uniform(min(vis_min, kend));          // turns that end here or before mask nothing
    const float sc = fmaxf(fabsf(a.scale) * kLog2eP, 1.17549435e-38f);

    floatx16 o[DT], ol;                                     // sums, and of the weights alone (rows all alike)
    const u32x4 ones{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
    float m;
    auto start = [&] {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            ol[i] = 0.f;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t][i] = 0.f;
        }
        m = -INFINITY;
    };
    start();
    if (tid == 0) s_met = 0;

    // A wave without rows stages its share only (256 groups of 132 rows: 106.6 us, then 100.8).
    auto attend = [&](auto works, auto with_care) {
        constexpr bool WORKS = decltype(works)::value, CARE = decltype(with_care)::value;
        int slot = 0;                                           // of s_bad, of the turn that is staged next
        for (int seg = kbeg; seg < kend; seg += segment) {
            const int seg_end = min(seg + segment, kend);
            if (seg > kbeg || a.splits > 1) id = table_entry(a, b, seg >> a.c.log_page);
            if (seg > kbeg) __syncthreads();                    // the pages of the segment before are used up
            look_up(seg, seg_end, id);
            stage(seg, s_stage[0], s_bad[slot], with_care);
            for (int k0 = seg, buf = 0; k0 < seg_end; k0 += KS, buf ^= 1) {
                const bool more = k0 + KS < seg_end;
                lds_barrier();                                  // the turn is staged; the one before is used up
                if (more) load(k0 + KS);
                [[maybe_unused]] const uint32_t *const bad = s_bad[slot];
                if constexpr (CARE) {
                    slot = slot == 2 ? 0 : slot + 1;
                    if (tid < 2) s_bad[slot == 2 ? 0 : slot + 1][tid] = 0;
                }
                if constexpr (WORKS) {
                    const u32x4 *keys = reinterpret_cast<const u32x4 *>(s_stage[buf]) + lane;
                    const u32x4 *values = reinterpret_cast<const u32x4 *>(s_stage[buf] + kValuesAt) + lane;
                    floatx16 st[KT];
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) st[t][i] = 0.f;
#pragma unroll
                    for (int c = 0; c < DS; ++c)
#pragma unroll
                        for (int t = 0; t < KT; ++t) st[t] = mfma32(keys[(t * DS + c) * 64], qf[c], st[t]);
                    if (k0 + KS > clear || any_none) {
#pragma unroll
                        for (int t = 0; t < KT; ++t) {
                            const int kb = k0 + 32 * t + 16 * gh;   // this lane's first key of the tile
                            const int real = page_of(kb).x >= kNone ? 0 : min(max(kend - kb, 0), 16);
                            const int top = min(max(vis - kb, 0), real);
                            uint32_t see = (1u << top) - 1u;
                            if (a.parent && live) see |= window16(s_anc[r], kb - s.lc) & ((1u << real) - 1u);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (!(see >> i & 1)) st[t][i] = -INFINITY;
                        }
                    }
                    if constexpr (CARE) {
#pragma unroll
                        for (int t = 0; t < KT; ++t) {
                            const uint32_t in = bad[t] >> (16 * gh);    // this lane's keys of the tile
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if ((in >> i & 1u) && st[t][i] != -INFINITY) st[t][i] = NAN;
                        }
                    }
                    float bm = -INFINITY;
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) bm = fmaxf(bm, st[t][i]);
                    {
                        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(bm), __float_as_uint(bm), false, false);
                        bm = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * sc;
                    }
                    const bool raise = bm > m + kLazyRescale;       // always when m is still -inf
                    if (__builtin_expect(__ballot(raise) != 0, 0)) {
                        const float alpha = raise ? __builtin_amdgcn_exp2f(m - bm) : 1.f;   // 0 from -inf
                        if (raise) m = bm;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            ol[i] *= alpha;
#pragma unroll
                            for (int t = 0; t < DT; ++t) o[t][i] *= alpha;
                        }
                    }
                    // a query that has seen nothing yet keeps m = -inf and adds nothing
                    const float mm = m == -INFINITY ? INFINITY : m;
                    u32x4 pb[KT][2];
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int v = 0; v < 2; ++v)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                pb[t][v][i] = bf16_pair(__builtin_amdgcn_exp2f(fmaf(st[t][8 * v + 2 * i], sc, -mm)),
                                                        __builtin_amdgcn_exp2f(fmaf(st[t][8 * v + 2 * i + 1], sc, -mm)));
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            ol = mfma32(ones, pb[t][v], ol);
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32(values[((dt * KT + t) * 2 + v) * 64], pb[t][v], o[dt]);
                        }
                }
                if (more) stage(k0 + KS, s_stage[buf ^ 1], s_bad[slot], with_care);
            }
        }
    };
    const bool idle = __ballot(live) == 0;
    if (idle) attend(std::false_type{}, std::false_type{});
    else attend(std::true_type{}, std::false_type{});
    if (all_see < kend) {
        __syncthreads();
        if (__builtin_expect(uniform(s_met), 0)) {          // once more, with care
            if (tid < 6) s_bad[tid / 2][tid % 2] = 0;
            start();
            id = table_entry(a, b, kbeg >> a.c.log_page);
            attend(std::true_type{}, std::true_type{});
        }
    }

    if (!valid) return;
    // O^T tile t, elements 4e .. 4e + 3: d = 32 t + 8 e + 4 gh + 0..3 of this lane's query
    const float l = live ? ol[0] : 0.f;                     // no query: unmasked turns gave it some weights
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = live ? o[t][i] : 0.f;
    if (cut.pieces == 1) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;   // NaN stays
        char *dst = static_cast<char *>(a.out) + (R * D + 4 * gh) * 2;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<u32x2 *>(dst + (32 * t + 8 * e) * 2) =
                    u32x2{bf16_pair(o[t][4 * e] * inv, o[t][4 * e + 1] * inv), bf16_pair(o[t][4 * e + 2] * inv, o[t][4 * e + 3] * inv)};
    } else {
        const int64_t at = w.piece * (static_cast<int64_t>(a.B) * a.n_q * a.Hq) + R;
        float *po = a.part_o + at * D + 4 * gh;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<floatx4 *>(po + 32 * t + 8 * e) =
                    floatx4{o[t][4 * e], o[t][4 * e + 1], o[t][4 * e + 2], o[t][4 * e + 3]};
        if (gh == 0) a.part_ml[at] = make_float2(live ? m : -INFINITY, l);
    }
}

// Joins the pieces of the rows that were cut: one wave per query row, lane s weighs piece s,
// then D / 4 lanes take one piece's columns, four each, 64 / (D / 4) pieces side by side.
template <int D>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
    constexpr int LP = D / 4, SP = 64 / LP, U = 4;
    const int lane = threadIdx.x & 63;
    const int64_t rows_all = static_cast<int64_t>(a.B) * a.n_q * a.Hq;
    const int64_t R = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (R >= rows_all) return;
    const int b = quot(a.by_seq_rows, static_cast<uint32_t>(R));
    const uint32_t pos = quot(a.by_hq, static_cast<uint32_t>(R));
    const int r = pos - static_cast<uint32_t>(b) * a.n_q, hq = static_cast<uint32_t>(R) - pos * a.Hq;
    const int c = lane % LP, sp = lane / LP;
    // the first pieces' sums are asked for before the sequence's length says how many there are
    // (what no piece has written is not used)
    float2 ml = a.part_ml[min(lane, a.splits - 1) * rows_all + R];
    floatx4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        v[u] = *(reinterpret_cast<const floatx4 *>(a.part_o + (min(u * SP + sp, a.splits - 1) * rows_all + R) * D) + c);
    const int grp = a.by_grp.d, tile = 16 * a.row_tiles * a.row_waves;
    const int qi = r * grp + hq % grp, q0 = qi / tile * tile;
    const Cut cut = cut_of(a, sequence_of(a, b), q0, min(q0 + tile, a.n_q * grp));
    if (cut.pieces == 1) return;                            // written whole
    const int n = cut.pieces;
    if (lane >= n) ml = make_float2(-INFINITY, 0.f);
    float M = ml.x;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float l = w * ml.y;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += SP * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * SP + sp;
            const float ws = __shfl(w, s & 63);
            const bool in = s < n;
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] = in ? fmaf(ws, v[u][k], acc[k]) : acc[k];
        }
        if (s0 + SP * U < n) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                v[u] = *(reinterpret_cast<const floatx4 *>(a.part_o + (min(s0 + (U + u) * SP + sp, n - 1) * rows_all + R) * D) + c);
        }
    }
#pragma unroll
    for (int off = LP; off < 64; off <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], off);
    if (sp == 0) {
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
        const u32x2 q{bf16_pair(acc[0] * inv, acc[1] * inv), bf16_pair(acc[2] * inv, acc[3] * inv)};
        *reinterpret_cast<u32x2 *>(static_cast<char *>(a.out) + (R * D + 4 * c) * 2) = q;
    }
}

// Up to 16 rows of a group, whose keys are read by one workgroup only: not kept in the caches where every
// load takes whole 64-byte runs of keys and of values, as with e4m3 pages of 64 places.  64 single tokens
// at about 3600 positions: kept 86.4 us, not kept 80.1; pages of 128, 128 tokens 168.6 and 191.7 (the
// other half of a run is fetched again); of 16, 48 tokens 76.5 and 77.3; bf16 178 and 202.
// Where several workgroups of up to 16 rows share a group (small calls spread theirs) they read the same keys,
// which are then kept: one sequence of 334 positions and 17 queries 8.03 us, not kept 8.27; of 1511 and 11
// queries 12.2 and 12.6; a tree of 60 nodes after 450 positions 10.1 and 10.4.
constexpr int kNontemporalPage = 6;   // log2 of its places

template <int D, bool F8>
void run_attention(const PagedArgs &a, unsigned grid, hipStream_t s) {
    const dim3 g(grid), t(kThreads);
    if (a.row_waves == 4) hipLaunchKernelGGL((k_paged_attention_wide<D, F8>), g, t, 0, s, a);
    else if (a.row_waves == 2 && a.row_tiles == 3) hipLaunchKernelGGL((k_paged_attention<D, F8, 3, 2>), g, t, 0, s, a);
    else if (a.row_waves == 2) hipLaunchKernelGGL((k_paged_attention<D, F8, 2, 2>), g, t, 0, s, a);
    else if (a.row_tiles == 3) hipLaunchKernelGGL((k_paged_attention<D, F8, 3, 1>), g, t, 0, s, a);
    else if (a.row_tiles == 2) hipLaunchKernelGGL((k_paged_attention<D, F8, 2, 1>), g, t, 0, s, a);
    else if (F8 && a.c.log_page == kNontemporalPage && a.by_blocks.d == 1)
        hipLaunchKernelGGL((k_paged_attention<D, F8, 1, 1, F8>), g, t, 0, s, a);
    else hipLaunchKernelGGL((k_paged_attention<D, F8, 1, 1>), g, t, 0, s, a);
}

constexpr int64_t kCus = 256;         // compute units of an MI355X

}  // namespace

PagedPlan paged_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq) {
    PagedPlan p{1, 1, 0, 1, kMinPiece, static_cast<int64_t>(B) * n_q * Hq, 0};
    const int64_t tiles = (static_cast<int64_t>(n_q) * (Hq / c.H) + 15) / 16;
    if (B <= 0 || tiles == 0) return p;
    // The lengths are on the device: the rules below go by the table's room, so the figures are of tables
    // cut to the sequences.  With room for 32768 positions few short sequences get larger workgroups, pieces that stay
    // empty and a join with nothing to join: one sequence of 334 positions 8.2 us and 19.4, a token after
    // 300 8.5 and 13.9, a tree of 38 nodes after 1000 positions 12.5 and 20.1.
    const int64_t groups = static_cast<int64_t>(B) * c.H, room = static_cast<int64_t>(c.max_pages) << c.log_page;
    const int64_t pieces = (room + kMinPiece - 1) / kMinPiece;
    int64_t per_block = 0;                                  // row tiles of a workgroup
    // Small calls: as few rows a workgroup as give every CU at most one, cut over the keys too.  One
    // sequence of 317 positions, 68 rows a group: 16 rows 8.0 us, 32 10.2, 48 13.1; a tree of 38 nodes after 1000
    // positions 12.5, 13.8 and 15.6; two sequences of 2017 positions 16.8, 15.2 and 17.7.
    for (int rt = 1; rt <= kMaxRowTiles && !per_block; ++rt)
        if (groups * ((tiles + rt - 1) / rt) * pieces <= kCus) per_block = p.row_tiles = rt;
    if (!per_block) {
        // With over three tiles two waves of up to three share keys where that makes a workgroup for every CU (68
        // rows in 512 groups: 65.7 us, as two workgroups that share nothing 77; in 16 groups 45 and 29.8).  Over six
        // tiles the wide kernel's cost less each, but it takes them by eight: sharing waves where they take
        // under four fifths as many.  Of 32 + 2000 positions, 288 groups, e4m3: 132 to 188 rows 81 to 83 us and
        // wide 101 to 102, 276 rows 102 and 123; bf16 108 to 111 and 111 to 117, 127 and 140; 100 rows (as many tiles) 85.1 and
        // 85.6; 124 rows of bf16 as two workgroups 90, wide 63.  128 groups of 164 rows 40.2 and 51.1, 64 31.9 and 31.2.
        const int64_t pairs = (tiles + 2 * kMaxRowTiles - 1) / (2 * kMaxRowTiles);
        const int64_t shared = pairs * 2 * ((tiles + 2 * pairs - 1) / (2 * pairs)), wide = (tiles + 7) / 8 * 8;
        if (tiles > kMaxRowTiles && groups * pairs >= kCus && (pairs == 1 || 5 * shared < 4 * wide)) p.row_waves = 2;
        else if (tiles > 2 * kMaxRowTiles) p.row_waves = 4;
        // rows shared out evenly over the fewest workgroups
        const int64_t most = p.row_waves == 4 ? kWideRows / 16 : kMaxRowTiles * p.row_waves, blocks = (tiles + most - 1) / most;
        p.row_tiles = p.row_waves == 4 ? kWideRows / 64 : static_cast<int32_t>((tiles + blocks * p.row_waves - 1) / (blocks * p.row_waves));
        per_block = p.row_tiles * p.row_waves;
    }
    p.blocks = static_cast<int32_t>((tiles + per_block - 1) / per_block);
    const int64_t units = groups * p.blocks;
    p.min_piece = p.row_waves == 4 ? kMinPieceWide : kMinPiece;
    // Cut only while that fills CUs: each has two workgroups then.  16 x 8 groups in two blocks, 1037
    // positions: uncut 17.3 us, in two pieces 24.6; 8 x 17 blocks, 515 positions 19.1 and 27.6; 16 groups in two
    // blocks, 16401 positions: 8 pieces 35.0, 16 pieces 29.8.
    if (units <= kCus / 2)
        p.splits = static_cast<int32_t>(std::max<int64_t>(
            std::min({2 * kCus / units, (room + p.min_piece - 1) / p.min_piece, kMaxPieces}), 1));
    p.grid = (groups * p.splits + kXcds - 1) / kXcds * kXcds * p.blocks;     // each XCD takes as many
    return p;
}

hipError_t launch_paged_attention(PagedArgs a, const PagedPlan &p, hipStream_t s) {
    a.row_tiles = p.row_tiles;
    a.row_waves = p.row_waves;
    a.splits = p.splits;
    a.min_piece = p.min_piece;
    a.by_grp = fast_div(a.Hq / a.c.H);
    a.by_blocks = fast_div(p.blocks);
    a.by_heads = fast_div(a.c.H);
    a.by_splits = fast_div(p.splits);
    a.by_seq_rows = fast_div(static_cast<uint32_t>(a.n_q) * static_cast<uint32_t>(a.Hq));
    a.by_hq = fast_div(a.Hq);
    const unsigned grid = static_cast<unsigned>(p.grid);
    if (a.c.D == 128) a.c.f8 ? run_attention<128, true>(a, grid, s) : run_attention<128, false>(a, grid, s);
    else a.c.f8 ? run_attention<64, true>(a, grid, s) : run_attention<64, false>(a, grid, s);
    if (p.splits > 1) {
        const dim3 jgrid(static_cast<unsigned>((p.rows + 3) / 4));
        if (a.c.D == 128) hipLaunchKernelGGL(k_paged_join<128>, jgrid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(k_paged_join<64>, jgrid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace cospec
