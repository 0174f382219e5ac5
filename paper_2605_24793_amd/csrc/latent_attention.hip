// Attention over the paged cache of latent vectors, in the absorbed form: all heads' queries meet
// the same vectors, which are keys and values at once.
//
//   s_j = scale (q . c_j + q' . r_j),   o = sum_j softmax(s)_j c_j
//
// One pass over the positions.  A sequence's rows (query positions x heads) share all of its keys, so a position of
// 2 (dc + 64) bytes serves 2 (2 dc + 64) operations for every row: from about 128 rows on the matrix cores bound
// it, below the memory.
#include <algorithm>
#include <type_traits>

#include "attend.h"
#include "latent.h"
#include "turn_flags.h"

namespace cospec {
namespace {

constexpr int kFewRows = 32, kManyRows = 64;   // of a workgroup
constexpr int kRotBytes = kRotated * 2;

// Keys of a piece, at least, where there are up to 16 pieces, and beyond.  Short pieces save turns, but the join reads every
// one of them.  A query of 16 heads after 2000 positions (e4m3, d_c = 512): 16 pieces of 128 keys 13.2 us, 8 of 256 14.3, 4
// of 512 18; after 8000 positions 63 of 128 17.0, 32 of 256 15.8; four queries of 32 heads after 4000 positions 32 of 128
// 17.7, 16 of 256 16.3.
constexpr int kMinPieceLatent = 128, kMinOfManyPieces = 256;
constexpr int64_t kFewPieces = 16;

constexpr float kFar = 60.f;          // log2 units a score may exceed a row's m by (weights and sums are floats)

// A latent's sixteen-byte pieces lie in LDS in another order: piece i at place i ^ turned(key), sixteen at a time, so that
// neither product's reads meet in the 64 banks: the first one's, sixteen rows' same piece, and the second one's, two
// pieces of eight rows (e4m3) or four of four (bf16).  Rotated keys, eight pieces each, likewise.  (Of the whole kernel's LDS
// cycles 10% are conflicts all the same over e4m3, 34% over bf16 of 512 components.)
template <bool F8> __device__ inline int turned(int key) {
    return F8 ? (key & 7) << 1 | (key >> 3 & 1) : (key & 3) << 2 | (key >> 2 & 3);
}

__device__ inline int turned_rotated(int key) { return key >> 1 & 7; }

// A wave's part of a turn, SR keys from `first` on (all of one page), on its way into LDS.
template <int DC, bool F8, int SR> struct TurnLoads {
    static constexpr int RB = DC * (F8 ? 1 : 2), RPI = 1024 / RB, PPR = RB / 16;   // rows of a load, pieces of a row
    static constexpr int NC = SR / RPI, NR = SR / 8;        // loads of latents, of rotated keys
    static constexpr int COUNT = NC + NR + (F8 ? 1 : 0);
    uint32_t c_off[NC], r_off[NR];
    int first;

    __device__ inline void begin(int lane, int first_key) {
        first = first_key;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int row = lane / PPR;
            c_off[i] = row * RB + ((lane % PPR) ^ turned<F8>(first + i * RPI + row)) * 16;
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int row = lane / 8;
            r_off[i] = row * kRotBytes + ((lane % 8) ^ turned_rotated(first + i * 8 + row)) * 16;
        }
    }
    // The page of a turn's keys, or page 0 (what is no key of the sequence is not used).
    __device__ inline uint32_t page(const PageArgs &c, const int32_t *row, int k0, int kend) const {
        const uint32_t id = scalar_load(row + (min(k0 + first, kend - 1) >> c.log_page));
        return id < static_cast<uint32_t>(c.n_pages) ? id : 0u;
    }
    __device__ inline void load(const PageArgs &c, uint32_t page, int k0, uint32_t stage, int rot_at, int scale_at, int lane) const {
        const int64_t place = (static_cast<int64_t>(page) << c.log_page) + ((k0 + first) & ((1 << c.log_page) - 1));
        load_lds_rows<NC>(c.k + place * RB, c_off, stage + first * RB);
        load_lds_rows<NR>(c.v + place * kRotBytes, r_off, stage + rot_at + first * kRotBytes);
        if (F8 && lane < SR) load_lds4(reinterpret_cast<const char *>(c.k_scale + place), lane * 4, stage + scale_at + first * 4);
    }
};

// Which unit a workgroup takes, and which piece of its keys.  Whole units come first.  Workgroups are dealt to the
// XCDs round-robin: each XCD takes consecutive units, which are blocks of the same sequences and read the
// same keys from its L2; a sequence's last rows, which see the most keys, come first.
struct Unit {
    int b, block, piece;
    int cut;                   // among the units that are cut, or -1: whole
};

__device__ inline Unit unit_at(const LatentArgs &a, int u, int piece, int cut) {
    const int b = quot(a.by_blocks, u);
    return Unit{b, static_cast<int>(a.by_blocks.d) - 1 - (u - b * static_cast<int>(a.by_blocks.d)), piece, cut};
}

__device__ inline Unit unit_of_workgroup(const LatentArgs &a) {
    const int w = blockIdx.x;
    if (w < a.whole) return unit_at(a, w % kXcds * (a.whole / kXcds) + w / kXcds, 0, -1);
    const int cut = quot(a.by_splits, w - a.whole), piece = w - a.whole - cut * a.splits;
    return unit_at(a, a.whole + cut, piece, a.splits > 1 ? cut : -1);
}

__device__ inline Cut cut_of_unit(const LatentArgs &a, const Unit &u, const Seq &s, int q0, int q1) {
    Cut c = cut_of(a, s, q0, q1);
    if (u.cut < 0) c.chunk = c.kend, c.pieces = 1;
    return c;
}

// The workspace's row of a unit's row, in its piece.
__device__ inline int64_t part_row(const LatentArgs &a, const Unit &u, int row, int rows) {
    return (static_cast<int64_t>(u.cut) * a.splits + u.piece) * rows + row;
}

// A lane's part of a row's sums into LDS: tile dt, elements 4e .. 4e + 3 are the components 32 dt + 8 e + 0..3 from `dst`
// on.  Whole rows are divided by the weights' sum L; pieces are kept as they are.
template <int DT> __device__ inline void put_rows(const floatx16 (&o)[DT], float L, char *dst) {
    const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;   // NaN stays
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            floatx4 x;
#pragma unroll
            for (int y = 0; y < 4; ++y) x[y] = L == 0.f ? 0.f : o[dt][4 * e + y] * inv;
            *reinterpret_cast<u32x2 *>(dst + (32 * dt + 8 * e) * 2) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
        }
}

template <int DT> __device__ inline void put_sums(const floatx16 (&o)[DT], char *dst) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            *reinterpret_cast<floatx4 *>(dst + (32 * dt + 8 * e) * 4) =
                floatx4{o[dt][4 * e], o[dt][4 * e + 1], o[dt][4 * e + 2], o[dt][4 * e + 3]};
}

// Rows in LDS, `stride` bytes apart, to memory at `to`, where they lie one after the other.
template <int ROW_BYTES, int T> __device__ inline void store_rows(const char *from, int stride, int rows, char *to, int tid) {
    constexpr int PR = ROW_BYTES / 16;
    asm volatile("" : "+v"(tid));                           // (addresses are found here, and not kept through the loop before)
    for (int i = tid; i < rows * PR; i += T) {
        const int r = i / PR, p = i % PR;
        *reinterpret_cast<u32x4 *>(to + static_cast<int64_t>(i) * 16) = *reinterpret_cast<const u32x4 *>(from + r * stride + p * 16);
    }
}

// Makes zeros of a staged turn's latents that hold no key of the sequence (such places may hold anything, and a
// weight of zero does not make a NaN harmless), and of elements that are not finite, whose keys are marked in `bad`.
// By all T threads, between barriers.
template <int RB, int KS, int T, bool F8>
__device__ inline void clean_turn(char *stage, float *scales, uint32_t *bad, int tid, bool real) {
    constexpr int PT = T / KS;                              // threads of a key, of one wave
    const int key = tid / PT, part = tid % PT;
    uint32_t top = 0;
#pragma unroll 2
    for (int i = 0; i < RB / 16 / PT; ++i) {
        u32x4 *at = reinterpret_cast<u32x4 *>(stage + key * RB + (part + PT * i) * 16);
        u32x4 x = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t t = not_finite<F8>(x[e], 0x01010101u);
            top |= t;
            x[e] = real ? x[e] & ~(t | (t - (t >> (F8 ? 7 : 15)))) : 0u;
        }
        *at = x;
    }
    bool marked = top != 0;
    if constexpr (F8) {
        const float sv = scales[key];
        const bool wild = !(fabsf(sv) < INFINITY);
        marked |= wild;
        wait_lds();
        if (part == 0 && (wild || !real)) scales[key] = 0.f;
    }
    if (real && marked) atomicOr(&bad[key >> 5], 1u << (key & 31));
}

// A workgroup's queries (ROWS rows that lie one after the other in memory) on their way into LDS, by T threads: a lane of a
// product reads a row's pieces, which from memory would take a line for each.  Piece p of row r lies at place
// p ^ turned_rotated(r) of its eight.
template <int DC, int ROWS, int T> __device__ inline void load_queries(const char *rows_at, int rows, uint32_t to, int wave, int lane) {
    constexpr int QB = (DC + kRotated) * 2, PQ = QB / 16, LOADS = ROWS * QB / 1024, N = (LOADS + T / 64 - 1) / (T / 64);
    static_assert(ROWS * QB % 1024 == 0 && PQ % 8 == 0 && QB % 256 == 128);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = (wave * N + i) * 64 + lane, r = at / PQ, p = (at - r * PQ) ^ turned_rotated(r);
        if (LOADS % (T / 64) == 0 || wave * N + i < LOADS)
            load_lds16<false>(rows_at + static_cast<int64_t>(min(r, rows - 1)) * QB + p * 16, to + (wave * N + i) * 1024);
    }
}

template <int DC> __device__ inline u32x4 query_piece(const char *queries, int row, int piece) {
    constexpr int QB = (DC + kRotated) * 2;
    return *reinterpret_cast<const u32x4 *>(queries + row * QB + (piece ^ turned_rotated(row)) * 16);
}

// A workgroup takes up to 64 rows of a sequence (or 32, where there are no more), and all its keys or a piece of them, with
// four waves for the scores and four for the sums, one of each on a SIMD.  While the latter add up one turn, the
// former work on the next, so that the matrix cores are fed by one wave while the other is at its exponentials,
// conversions or waits.  (One wave for both leaves them idle then: a lone wave issues a vector instruction every 7.5
// cycles.  Two for both would need 144 registers of queries and 64 of sums each, and room to work.)
//
// S^T = K Q^T and O^T = C^T P^T: the second product's operand C^T has positions where the rows lie; LDS turns
// them while they are read (ds_read_b64_tr).  Scores: a part of a turn's keys and of the rows a wave, with products of
// 32 x 32 (64 rows, turns of 64 keys) or 16 x 16.  Sums: all rows and a quarter of the components a wave.  The
// rounded weights go from one to the other through LDS.
//
// After barrier i turn i is staged and turn i - 1 weighed: the scores' waves take turn i, the sums' waves turn
// i - 1, and load ahead.
//
// A row's weights are 2^(s - m) with m the maximum of the first turn in which it sees a key: that is as exact as with
// the running one, as long as no later score is kFar above it.  Then the sums need not be scaled
// down on the way, and all waves know m.  Where a score is, the piece is taken again: its maxima first, then the
// sums (the rest of the pass that finds it is for nothing: nothing else may leave the loop, or the compiler
// keeps the sums twice).
//
// 64 rows: a turn of 64 e4m3 keys takes 3100 cycles, its products 2176 (clocks read in a copy of the kernel; the sums' waves
// take 900 to get its loads out, and between products they take as long and come later: 160 us where this takes 149), and each
// workgroup's start and end 20 000; counted over a whole call the matrix cores are at work half of the CUs' cycles.  64 x 17
// queries of 32 heads after 1536 to 2048 e4m3 positions 155 to 159 us from card to card, 859 to 883 TFLOP/s; 16 trees of 60
// nodes over bf16 138 us, 874.  Turns of 32 e4m3 keys took 178 us where those of 64 took 157; bf16 of 512 components has no
// room for three turns of 64.
// 32 rows: a workgroup has few products and waits for loads, so turns are short and four are on their way: 64 x 1 query of
// 32 heads after up to 4096 e4m3 positions 47 us, 3.3 TB/s with the join (turns of 64 keys, one on its way: 48.5 where these
// took 46.3; five of 32: 46.7).  The loads reach 4.2 TB/s, which is not the memory's limit: one workgroup fills a CU, and nothing
// covers its start and end.  Over bf16 64.5 us, 5.0 TB/s.  The other choice: these with 64 rows, half of them empty, 50.8 us;
// 64 x 17 queries by workgroups of 32 rows 201 us for 151, 64 x 2 after 2048 positions 42.8 for 36.4.
template <int DC, bool F8, int ROWS>
__global__ __launch_bounds__(512, 1) void k_latent_attention(LatentArgs a) {
    constexpr int EB = F8 ? 1 : 2, RB = DC * EB;            // bytes of a latent
    constexpr int KS = RB > 512 || ROWS == 32 ? 32 : 64;    // keys of a turn
    constexpr bool WIDE = KS == 64 && ROWS == 64;           // scores by 32 x 32 products, or by 16 x 16
    constexpr int QW = WIDE ? 32 : 16, TK = QW;             // rows and keys of a tile of scores
    constexpr int KP = KS / TK, RP = 4 / KP;                // parts of the keys, and of the rows, among the scores' waves
    constexpr int QT = ROWS / RP / QW;                      // tiles of a wave
    constexpr int SK = WIDE ? 16 : 32;                      // components of a k-step of its products
    constexpr int CS = DC / SK, RS = kRotated / SK;         // its k-steps, of latents and of rotated keys
    constexpr int NS = WIDE ? 16 : 4;                       // scores of a lane and query tile
    constexpr int DT = DC / 4 / 32, RT = ROWS / 32;         // component tiles, and tiles of rows, of a sums' wave
    constexpr int kRotAt = KS * RB, kScaleAt = kRotAt + KS * kRotBytes, kStage = kScaleAt + (F8 ? KS * 4 : 0);
    constexpr int NB = RB > 512 ? 4 : ROWS == 32 ? 6 : 3, AHEAD = NB - 2;   // turns in LDS, and on their way
    constexpr int PPR = RB / 16;                            // pieces of a row
    constexpr int SR = KS / 4;                              // keys that a sums' wave loads
    constexpr int LPT = TurnLoads<DC, F8, SR>::COUNT;       // its loads of a turn
    constexpr int kWeightRow = KS * 2 + 16;                 // bytes
    __shared__ __attribute__((aligned(256))) char s_ring[NB * kStage];
    __shared__ __attribute__((aligned(16))) char s_weight[2][ROWS * kWeightRow];
    __shared__ uint32_t s_page[kThreads];
    __shared__ uint32_t s_seen[ROWS][8];                    // ancestors of the rows' nodes
    __shared__ float s_max[KP][ROWS];
    __shared__ float s_sum[KP][ROWS];
    __shared__ uint32_t s_bad[2];                           // of a turn's keys: latent or scale not finite
    __shared__ TurnFlags s_new;                             // a row's first keys, or a score far above its m
    __shared__ int s_far, s_none;

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int gh = lane >> 5, l32 = lane & 31;
    const int rows = a.n_q * a.Hq;
    const Unit w_ = unit_of_workgroup(a);
    const int b = w_.b;
    const int q0 = w_.block * ROWS, q1 = min(q0 + ROWS, rows);
    const int64_t R0 = static_cast<int64_t>(b) * rows;
    // the queries go behind the turns that are loaded before they are read
    char *const s_q = s_ring + AHEAD * kStage;
    static_assert(AHEAD * kStage + ROWS * (DC + kRotated) * 2 <= NB * kStage);
    load_queries<DC, ROWS, 512>(static_cast<const char *>(a.q) + (R0 + q0) * ((DC + kRotated) * 2), q1 - q0, uniform(lds_address(s_q)), wave, lane);
    const Seq s = sequence_of(a, b);
    const Cut cut = cut_of_unit(a, w_, s, q0, q1);
    if (w_.piece >= cut.pieces) {
        wait_vm<0>();                                       // (nothing may come into LDS that is another's then)
        return;
    }
    const int kbeg = w_.piece * cut.chunk, kend = min(kbeg + cut.chunk, cut.kend);
    const int all_see = seen_by_all(a, s, q0, kend);        // keys below are seen by every row that sees any
    if (a.parent) {
        uint32_t(*const anc)[8] = reinterpret_cast<uint32_t(*)[8]>(s_ring);
        find_ancestors(a, b, anc, reinterpret_cast<int *>(s_ring + kMaxSeqRows * 32));
        if (tid < ROWS * 8) s_seen[tid / 8][tid % 8] = anc[quot(a.by_grp, min(q0 + tid / 8, q1 - 1))][tid % 8];
        __syncthreads();
    }
    if (tid == 0) s_new.lower_all(), s_far = 0;
    wait_vm<0>();
    __syncthreads();                                        // the queries are there

    const int segment = kSegment << a.c.log_page;
    const uint32_t ring = uniform(lds_address(s_ring));
    const float sc = fmaxf(fabsf(a.scale) * kLog2eP, 1.17549435e-38f);

    auto joined_max = [&](int row) {
        float x = s_max[0][row];
#pragma unroll
        for (int i = 1; i < KP; ++i) x = fmaxf(x, s_max[i][row]);
        return x;
    };
    auto joined_sum = [&](int row) {
        float x = s_sum[0][row];
#pragma unroll
        for (int i = 1; i < KP; ++i) x += s_sum[i][row];
        return x;
    };

    // All of it, as one kind of wave does it: both meet the same barriers.
    auto work = [&](auto kind) __attribute__((always_inline)) {
        constexpr bool SCORES = decltype(kind)::value;
        // scores: queries, in the order in which the keys' pieces come (of e4m3 a lane's sixteen bytes are two k-steps)
        const int ql = WIDE ? l32 : lane & 15, kg = WIDE ? gh : lane >> 4;   // query, k-piece
        const int rw = (wave & 3) % RP, kp = (wave & 3) / RP;
        [[maybe_unused]] u32x4 qf[QT][CS + RS];
        [[maybe_unused]] int node[QT], vis[QT];             // keys [0, vis) are seen
        [[maybe_unused]] float m[QT];
        const int krow = kp * TK + ql;
        [[maybe_unused]] const uint32_t k_at = krow * RB + (kg ^ turned<F8>(krow)) * 16;
        [[maybe_unused]] const uint32_t r_at = kRotAt + krow * kRotBytes + (kg ^ turned_rotated(krow)) * 16;
        if constexpr (SCORES) {
            const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;   // scores as |scale| (+-q) . k: the largest product is the largest
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const int row = q0 + rw * (QT * QW) + t * QW + ql, qi = min(row, q1 - 1);
                node[t] = quot(a.by_grp, qi);
                const int64_t p = s.qs + node[t];
                const bool live = row < q1 && p >= 0 && p < s.end;
                vis[t] = !live ? 0 : a.parent ? s.lc : p >= s.lc ? s.end : static_cast<int>(p) + 1;
                if (!live) node[t] = -1;
                m[t] = -INFINITY;
#pragma unroll
                for (int c = 0; c < CS + RS; ++c) {
                    const int d = c >= CS ? DC + (c - CS) * SK + kg * 8 : F8 ? c / 2 * (2 * SK) + kg * 16 + c % 2 * 8 : c * SK + kg * 8;
                    qf[t][c] = query_piece<DC>(s_q, row - q0, d / 8);
#pragma unroll
                    for (int x = 0; x < 4; ++x) qf[t][c][x] = live ? qf[t][c][x] ^ flip : 0u;
                }
            }
        }
        // sums
        const int pw = wave & 3;
        [[maybe_unused]] uint32_t v_at = 0;
        if constexpr (!SCORES) {
            const int j = lane & 15, cg = lane >> 4 & 1, row = 8 * gh + (F8 ? j >> 1 : j >> 2);
            const int piece = pw * (PPR / 4) + (F8 ? cg : 2 * cg + (j >> 1 & 1));
            v_at = row * RB + (piece >> 4) * 256 + ((piece ^ turned<F8>(row)) & 15) * 16 + (j & 1) * 8;
        }
        int first_page = 0, last_page = 0;                  // of those in LDS
        bool any_none = false;
        auto page_of = [&](int key) { return s_page[min(key >> a.c.log_page, last_page) - first_page]; };
        const int32_t *const pages = a.c.table + static_cast<int64_t>(b) * a.c.max_pages;
        [[maybe_unused]] TurnLoads<DC, F8, SR> loads;
        if constexpr (!SCORES) loads.begin(lane, pw * SR);
        [[maybe_unused]] auto load = [&](uint32_t page, int k0, int buf) {
            loads.load(a.c, page, k0, ring + buf * kStage, kRotAt, kScaleAt, lane);
        };

        // Once, unless a score lies far above its row's m: then once more for the maxima alone, and again for the sums.
        bool finding = false;
        [[maybe_unused]] bool met = false;                  // a turn without a mask: live rows see all of its keys
        for (;;) {
            [[maybe_unused]] floatx16 o[RT][DT];
            [[maybe_unused]] float l[QT];                   // of this lane's keys alone
            if constexpr (SCORES) {
#pragma unroll
                for (int t = 0; t < QT; ++t) l[t] = 0.f;
            } else {
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[t][dt][i] = 0.f;
            }
            for (int seg = kbeg; seg < kend; seg += segment) {
                const int seg_end = min(seg + segment, kend), turns = (seg_end - seg + KS - 1) / KS;
                first_page = seg >> a.c.log_page;
                last_page = (seg_end - 1) >> a.c.log_page;
                const uint32_t entry = table_entry(a, b, first_page);
                __syncthreads();                            // the pages of the segment before are used up
                if (tid == 0) s_none = 0;
                __syncthreads();
                if (tid <= last_page - first_page) {        // a page that is none is read as page 0, and not used
                    const bool none = entry >= static_cast<uint32_t>(a.c.n_pages);
                    s_page[tid] = none ? kNone : entry;
                    if (none) s_none = 1;
                }
                __syncthreads();
                any_none = uniform(s_none) != 0;
                met |= !any_none && seg + KS <= all_see;
                [[maybe_unused]] uint32_t next = 0;         // the page that is loaded from next
                if constexpr (!SCORES) {
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
                        if (i < turns) load(loads.page(a.c, pages, seg + i * KS, kend), seg + i * KS, i);
                    next = loads.page(a.c, pages, seg + AHEAD * KS, kend);
                }
                [[maybe_unused]] typename std::conditional<WIDE, floatx16, floatx4>::type st[QT];
                [[maybe_unused]] float sv[F8 ? NS : 1];     // scales of this lane's keys
                [[maybe_unused]] float bm[QT], sum[QT];
                int buf = 0;                                // of turn i
                for (int i = 0; i <= turns; ++i, buf = buf + 1 == NB ? 0 : buf + 1) {
                    const int k0 = seg + i * KS;
                    if constexpr (!SCORES) {                // turn i has come
                        if (AHEAD > 3 && i + 3 < turns) wait_vm<3 * LPT>();
                        else if (AHEAD > 2 && i + 2 < turns) wait_vm<2 * LPT>();
                        else if (AHEAD > 1 && i + 1 < turns) wait_vm<LPT>();
                        else wait_vm<0>();
                    }
                    lds_barrier();
                    [[maybe_unused]] auto weigh = [&](int turn) __attribute__((always_inline)) {
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            // a query that has seen nothing yet keeps m = -inf and adds nothing
                            const float mm = m[t] == -INFINITY || finding ? INFINITY : m[t];
                            sum[t] = 0.f;
                            char *to = s_weight[turn & 1] + (rw * (QT * QW) + t * QW + ql) * kWeightRow + (kp * TK + 4 * kg) * 2;
#pragma unroll
                            for (int e = 0; e < NS / 4; ++e) {
                                float p[4];
#pragma unroll
                                for (int x = 0; x < 4; ++x) {
                                    p[x] = __builtin_amdgcn_exp2f(fmaf(st[t][4 * e + x], sc, -mm));
                                    sum[t] += p[x];
                                    if constexpr (F8) p[x] *= sv[4 * e + x];
                                }
                                *reinterpret_cast<u32x2 *>(to + e * 16) = u32x2{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3])};
                            }
                        }
                    };
                    if (__builtin_expect(uniform(s_new.raised(i - 1)), 0)) {
                        // the same maximum in all waves, then the weights of turn i - 1 again
                        if constexpr (SCORES) {
                            if (kg == 0) {
#pragma unroll
                                for (int t = 0; t < QT; ++t) s_max[kp][rw * (QT * QW) + t * QW + ql] = bm[t];
                            }
                        }
                        lds_barrier();
                        if constexpr (SCORES) {
                            if (tid == 0) s_new.lower(i - 1);
                            bool above = false;
#pragma unroll
                            for (int t = 0; t < QT; ++t) {
                                const int row = rw * (QT * QW) + t * QW + ql;
                                const float top = joined_max(row);
                                if (m[t] == -INFINITY) m[t] = top;
                                else above |= top > m[t] + kFar;
                            }
                            if (__ballot(above) != 0 && lane == 0) s_far = 1;
                            weigh(i - 1);
                        }
                        lds_barrier();
                    }
                    const bool masked = i < turns && (k0 + KS > all_see || any_none);   // the same in the whole workgroup
                    char *const stage = s_ring + buf * kStage;
                    if (masked) {
                        if (tid < 2) s_bad[tid] = 0;
                        lds_barrier();
                        const int key = k0 + tid / (512 / KS);
                        clean_turn<RB, KS, 512, F8>(stage, reinterpret_cast<float *>(stage + kScaleAt), s_bad, tid,
                                                    key < kend && page_of(key) < kNone);
                        lds_barrier();
                    }
                    if constexpr (SCORES) {
                        if (i > 0) {
#pragma unroll
                            for (int t = 0; t < QT; ++t) l[t] += sum[t];
                        }
                        if (i == turns) break;
                        // S^T.  Operands are read from LDS a group ahead of the products that take them.
                        constexpr int LP = WIDE ? 2 : 4, PER = 16 / LP;  // pieces of a key that a load's lanes take side by side
                        constexpr int LOADS = CS / (F8 ? 2 : 1), G = F8 ? 2 : 4, NG = LOADS / G;
#pragma unroll
                        for (int t = 0; t < QT; ++t)
#pragma unroll
                            for (int x = 0; x < NS; ++x) st[t][x] = 0.f;
                        u32x4 kf[2][G], rf[RS];
                        auto read_keys = [&](int g) __attribute__((always_inline)) {
#pragma unroll
                            for (int x = 0; x < G; ++x) {
                                const int c = g * G + x;
                                kf[g & 1][x] = *reinterpret_cast<const u32x4 *>(stage + (k_at ^ (c % PER * LP * 16)) + c / PER * 256);
                            }
                        };
                        auto multiply = [&](u32x4 k, int c) __attribute__((always_inline)) {
#pragma unroll
                            for (int t = 0; t < QT; ++t) {
                                if constexpr (WIDE) st[t] = mfma32(k, qf[t][c], st[t]);
                                else st[t] = mfma(k, qf[t][c], st[t]);
                            }
                        };
                        read_keys(0);
                        read_keys(1);
                        if constexpr (F8) {
#pragma unroll
                            for (int e = 0; e < NS / 4; ++e) {
                                const floatx4 x = *reinterpret_cast<const floatx4 *>(stage + kScaleAt + (kp * TK + 8 * e + 4 * kg) * 4);
#pragma unroll
                                for (int y = 0; y < 4; ++y) sv[4 * e + y] = x[y];
                            }
                        }
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int x = 0; x < G; ++x) {
                                const u32x4 raw = kf[g & 1][x];
                                const int c = g * G + x;
                                if constexpr (F8) {
                                    multiply(widen(raw[0], raw[1], 1.f), 2 * c);
                                    multiply(widen(raw[2], raw[3], 1.f), 2 * c + 1);
                                } else {
                                    multiply(raw, c);
                                }
                            }
                            __builtin_amdgcn_sched_barrier(0);
                            if (g + 2 < NG) {
                                read_keys(g + 2);
                            } else if (g + 2 == NG) {
#pragma unroll
                                for (int c = 0; c < RS; ++c) rf[c] = *reinterpret_cast<const u32x4 *>(stage + (r_at ^ (c * LP * 16)));
                            }
                        }
                        if constexpr (F8) {
#pragma unroll
                            for (int t = 0; t < QT; ++t)
#pragma unroll
                                for (int x = 0; x < NS; ++x) st[t][x] *= sv[x];
                        }
#pragma unroll
                        for (int c = 0; c < RS; ++c) multiply(rf[c], CS + c);
                        if (masked) {
                            const int kb = k0 + kp * TK;
                            uint32_t real = low_bits(kend - kb);
                            if (page_of(kb) >= kNone) real &= 0xffff0000u;
                            if (TK == 32 && page_of(kb + 16) >= kNone) real &= 0x0000ffffu;
                            const uint32_t bad = s_bad[kp * TK / 32] >> (kp * TK % 32 + 4 * kg);
#pragma unroll
                            for (int t = 0; t < QT; ++t) {
                                uint32_t see = low_bits(vis[t] - kb);
                                if (a.parent && node[t] >= 0) see |= window32(s_seen[rw * (QT * QW) + t * QW + ql], kb - s.lc);
                                see = (see & real) >> (4 * kg);
#pragma unroll
                                for (int x = 0; x < NS; ++x) {
                                    const int bit = 8 * (x / 4) + x % 4;
                                    const float y = (bad >> bit & 1) != 0 ? NAN : st[t][x];
                                    st[t][x] = (see >> bit & 1) != 0 ? y : -INFINITY;
                                }
                            }
                        }
                        bool fresh = false;                 // a row's first keys, or a score far above m
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            bm[t] = -INFINITY;
#pragma unroll
                            for (int x = 0; x < NS; ++x) bm[t] = fmaxf(bm[t], st[t][x]);
                            if constexpr (WIDE) {
                                const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(bm[t]), __float_as_uint(bm[t]), false, false);
                                bm[t] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])) * sc;
                            } else {
                                bm[t] = max_rows(bm[t]) * sc;
                            }
                            fresh |= bm[t] > m[t] + kFar;   // always when m is still -inf
                        }
                        weigh(i);
                        if (finding) {
#pragma unroll
                            for (int t = 0; t < QT; ++t) m[t] = fmaxf(m[t], bm[t]);
                        } else if (__ballot(fresh) != 0 && lane == 0) {
                            s_new.raise(i);
                        }
                    } else {
                        const int to = buf + AHEAD >= NB ? buf + AHEAD - NB : buf + AHEAD;
                        if (i + AHEAD < turns) load(next, k0 + AHEAD * KS, to);
                        next = loads.page(a.c, pages, k0 + (AHEAD + 1) * KS, kend);
                        if (i == 0) continue;
                        // O^T += C^T P^T of turn i - 1, sixteen keys at a time
                        const char *const held = s_ring + (buf == 0 ? NB - 1 : buf - 1) * kStage;
                        const char *const w_at = s_weight[(i - 1) & 1] + l32 * kWeightRow + gh * 16;
                        constexpr int NV = KS / 16;
                        u32x4 pb[2][RT], vf[2][DT];          // (e4m3: two words of each)
                        auto read = [&](int v) __attribute__((always_inline)) {
                            const char *const at = held + v * 16 * RB;
#pragma unroll
                            for (int t = 0; t < RT; ++t) pb[v & 1][t] = *reinterpret_cast<const u32x4 *>(w_at + t * (32 * kWeightRow) + v * 32);
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) {
                                if constexpr (F8) {
                                    const i32x2 raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(at + (v_at ^ (dt * 32))));
                                    vf[v & 1][dt][0] = raw[0];
                                    vf[v & 1][dt][1] = raw[1];
                                } else {
                                    const uint32_t here = v_at ^ (dt * 64);
                                    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + here)));
                                    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * RB + (here ^ 16))));
                                    vf[v & 1][dt] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                                }
                            }
                        };
                        read(0);
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            if (v + 1 < NV) read(v + 1);
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) {
                                const u32x4 raw = vf[v & 1][dt], c = F8 ? widen(raw[0], raw[1], 1.f) : raw;
#pragma unroll
                                for (int t = 0; t < RT; ++t) o[t][dt] = mfma32(c, pb[v & 1][t], o[t][dt]);
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
            __syncthreads();
            const bool far = uniform(s_far) != 0;
            if constexpr (SCORES) {
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    if constexpr (!WIDE) l[t] += __shfl_xor(l[t], 16);
                    l[t] += __shfl_xor(l[t], 32);
                    const int row = rw * (QT * QW) + t * QW + ql;
                    if (kg == 0) {
                        // (unmasked turns give padding rows some weights; a row that met only scores of minus infinity, as
                        // infinite latents make them, has none, and sums that are not finite)
                        s_sum[kp][row] = node[t] < 0 ? 0.f : met && m[t] == -INFINITY ? NAN : l[t];
                        s_max[kp][row] = node[t] >= 0 || finding ? m[t] : -INFINITY;
                    }
                }
            }
            __syncthreads();
            if (!finding && !far) {
                // O^T tile dt, elements 4e .. 4e + 3: components 32 dt + 8 e + 4 gh + 0..3 of the wave's quarter, of row l32
                // of tile t: through LDS, so that whole rows are stored
                if (cut.pieces == 1) {
                    constexpr int STRIDE = DC * 2 + 16;
                    static_assert(ROWS * STRIDE <= NB * kStage);
                    if constexpr (!SCORES) {
#pragma unroll
                        for (int t = 0; t < RT; ++t) {
                            const int row = t * 32 + l32;
                            put_rows<DT>(o[t], joined_sum(row), s_ring + row * STRIDE + (pw * (DC / 4) + 4 * gh) * 2);
                        }
                    }
                    __syncthreads();
                    store_rows<DC * 2, 512>(s_ring, STRIDE, q1 - q0, static_cast<char *>(a.out) + (R0 + q0) * (DC * 2), tid);
                } else {
                    constexpr int STRIDE = DC * 4 + 16;
                    static_assert(32 * STRIDE <= NB * kStage);
                    const int64_t at = part_row(a, w_, 0, ROWS);
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        if (t) __syncthreads();
                        if constexpr (!SCORES) put_sums<DT>(o[t], s_ring + l32 * STRIDE + (pw * (DC / 4) + 4 * gh) * 4);
                        __syncthreads();
                        const int here = min(q1 - q0 - t * 32, 32);
                        if (here > 0) store_rows<DC * 4, 512>(s_ring, STRIDE, here, reinterpret_cast<char *>(a.part_o + (at + t * 32) * DC), tid);
                    }
                    if (tid < q1 - q0) a.part_ml[at + tid] = make_float2(s_max[0][tid], joined_sum(tid));
                }
                return;
            }
            if constexpr (SCORES) {
                if (finding) {                              // every row's maximum, joined over the parts of the keys
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const int row = rw * (QT * QW) + t * QW + ql;
                        m[t] = joined_max(row);
                    }
                }
            }
            if (tid == 0) s_far = 0;                        // (read by all before the barrier above)
            finding = !finding;
        }
    };
    if (wave < 4) work(std::true_type{});
    else work(std::false_type{});
}

// Joins the pieces of the units that were cut.  It waits for memory, so a workgroup takes a row and has eight pieces' loads out
// at a time (16 heads, 32 pieces: 17.9 us for both launches with a wave a row and four pieces, 15.8 so); lane s weighs piece s, then each thread takes
// DC / 256 components of every piece.  A launch after the pieces' own: their order is the same every time.
template <int DC>
__global__ __launch_bounds__(256) void k_latent_join(LatentArgs a) {
    constexpr int EACH = DC / 256, AT_ONCE = 8;             // components of a thread; pieces whose loads are out together
    using part = typename std::conditional<EACH == 2, float2, float>::type;
    const int lane = threadIdx.x & 63;
    const int rows = a.n_q * a.Hq, unit_rows = a.row_tiles;
    const int cut = blockIdx.x / unit_rows, row = blockIdx.x - cut * unit_rows;   // (a power of two)
    const Unit u = unit_at(a, a.whole + cut, 0, cut);
    const int q0 = u.block * unit_rows, q1 = min(q0 + unit_rows, rows);
    if (q0 + row >= q1) return;
    const int64_t R = static_cast<int64_t>(u.b) * rows + q0 + row, at = part_row(a, u, row, unit_rows);
    float2 ml = a.part_ml[at + static_cast<int64_t>(min(lane, a.splits - 1)) * unit_rows];
    const Cut c = cut_of(a, sequence_of(a, u.b), q0, q1);
    if (c.pieces == 1) return;                              // written whole
    const int n = c.pieces;
    const part *from = reinterpret_cast<const part *>(a.part_o + at * DC) + threadIdx.x;
    const int64_t step = static_cast<int64_t>(unit_rows) * 256;
    float acc[2] = {0.f, 0.f};
    float w = 0.f, l = 0.f;
    for (int p0 = 0; p0 < n; p0 += AT_ONCE) {
        part v[AT_ONCE];
#pragma unroll
        for (int p = 0; p < AT_ONCE; ++p) v[p] = from[min(p0 + p, n - 1) * step];
        if (p0 == 0) {                                      // while the first ones come
            if (lane >= n) ml = make_float2(-INFINITY, 0.f);
            float M = ml.x;
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
            w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
            // (a piece without a maximum has a weight sum of 0, or of NaN where the row saw only scores that are NaN)
            l = ml.x == -INFINITY ? ml.y : w * ml.y;
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
        }
#pragma unroll
        for (int p = 0; p < AT_ONCE; ++p) {
            const float wp = __shfl(w, p0 + p);
            const bool none = p0 + p >= n || __shfl(ml.x, p0 + p) == -INFINITY;   // (its sums may be anything)
            if constexpr (EACH == 2) {
                acc[0] = none ? acc[0] : fmaf(wp, v[p].x, acc[0]);
                acc[1] = none ? acc[1] : fmaf(wp, v[p].y, acc[1]);
            } else {
                acc[0] = none ? acc[0] : fmaf(wp, v[p], acc[0]);
            }
        }
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    const uint32_t out = bf16_pair(acc[0] * inv, acc[1] * inv);
    char *const dst = static_cast<char *>(a.out) + R * DC * 2;
    if constexpr (EACH == 2) reinterpret_cast<uint32_t *>(dst)[threadIdx.x] = out;
    else reinterpret_cast<uint16_t *>(dst)[threadIdx.x] = static_cast<uint16_t>(out);
}

template <int DC, bool F8> void run_attention(const LatentArgs &a, unsigned grid, hipStream_t s) {
    if (a.row_tiles == kManyRows) hipLaunchKernelGGL((k_latent_attention<DC, F8, kManyRows>), dim3(grid), dim3(512), 0, s, a);
    else hipLaunchKernelGGL((k_latent_attention<DC, F8, kFewRows>), dim3(grid), dim3(512), 0, s, a);
}

}  // namespace

LatentPlan latent_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq) {
    LatentPlan p{};
    p.splits = 1;
    const int64_t rows = static_cast<int64_t>(n_q) * Hq;
    if (B <= 0 || rows == 0) return p;
    p.rows = rows <= kFewRows ? kFewRows : kManyRows;
    p.blocks = static_cast<int32_t>((rows + p.rows - 1) / p.rows);
    p.units = static_cast<int64_t>(B) * p.blocks;
    // A workgroup fills a CU, so units come in rounds of one for each; what is left over is cut into pieces that fill
    // the CUs once: in equally many each, whatever their lengths, and from 129 units on not at all (130 x 1 query 51 us, 128 x 1
    // 50).  (64 x 17 queries, 64 of 576 units left over: 166 us uncut, 153 cut on the same card; 64 x 1 query 89 and
    // 46; one query over 2000 positions 33 and 12.)
    p.whole = p.units / kCus * kCus;
    const int64_t left = p.units - p.whole, room = static_cast<int64_t>(c.max_pages) << c.log_page;
    const int64_t most = std::max(std::min((room + kMinPieceLatent - 1) / kMinPieceLatent, kFewPieces), (room + kMinOfManyPieces - 1) / kMinOfManyPieces);
    if (left > 0) p.splits = static_cast<int32_t>(std::max<int64_t>(std::min({kCus / left, most, kMaxPieces}), 1));
    p.grid = p.whole + left * p.splits;
    p.parts = p.splits > 1 ? left * p.splits * p.rows : 0;
    return p;
}

hipError_t launch_latent_attention(LatentArgs a, const LatentPlan &p, hipStream_t s) {
    a.row_tiles = p.rows;
    a.splits = p.splits;
    a.min_piece = kMinPieceLatent;
    a.whole = static_cast<int32_t>(p.whole);
    a.by_grp = fast_div(a.Hq);
    a.by_blocks = fast_div(p.blocks);
    a.by_splits = fast_div(p.splits);
    const unsigned grid = static_cast<unsigned>(p.grid);
    if (a.c.D == 512) a.c.f8 ? run_attention<512, true>(a, grid, s) : run_attention<512, false>(a, grid, s);
    else a.c.f8 ? run_attention<256, true>(a, grid, s) : run_attention<256, false>(a, grid, s);
    if (p.splits > 1) {
        const dim3 jgrid(static_cast<unsigned>((p.units - p.whole) * p.rows));
        if (a.c.D == 512) hipLaunchKernelGGL(k_latent_join<512>, jgrid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(k_latent_join<256>, jgrid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace cospec
