// Attention over the paged key/value cache: the arbitrator's hybrid attention and the
// attention of token-tree nodes, for any number of queries per sequence.
//
// Online softmax: with scores s_j = scale * q . k_j, a running max m and the sums
// l = sum_j 2^(s_j log2 e - m), o = sum_j 2^(s_j log2 e - m) v_j, one pass over the keys gives
// o / l; raising m multiplies both sums by 2^(m_old - m_new), and sums over disjoint keys are
// joined the same way.
//
// Work split: the query rows (position x head) that share a key/value head of a sequence form
// a group.  A workgroup takes up to 16 * RT rows of a group, and its waves take turns at the
// group's keys, 64 at a time, all rows each: a wave reads its keys and values straight from the
// pages into the registers that the matrix instructions take them from, once, with no LDS
// and no barrier on the way, and the waves' sums are joined through LDS at the end.
//
// S^T = K Q^T (v_mfma_f32_16x16x32_bf16): lane l holds query column l % 16, so the softmax of a
// query stays in four lanes.  Which key stands in which row of a product is free: row i of
// tile t is key 16 (i / 4) + 4 t + i % 4 of the 64, so that lane l's scores are the 16 keys
// 16 (l / 16) + 4 t + r, in order.  These are also, as they stand, a lane's share of the
// second product's operand P^T, and the values it needs for them are 16 keys in a row: with
// values kept [d][place] they are 16 (e4m3) or 32 (bf16) contiguous bytes.
//
// e4m3: v_cvt_scalef32_pk_bf16_fp8 widens two elements and applies the page's power of two;
// e4m3 has fewer bits than bf16, so nothing is rounded, and one conversion serves all rows.
#include "paged.h"

namespace cospec {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float floatx4;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;             // of a workgroup
constexpr int kStep = 64;             // keys of a wave's turn
// 16-row tiles of a workgroup, at most: what the registers hold of queries, scores and sums
constexpr int kMaxRowTiles = 3;
constexpr int kMinPiece = 256;        // keys of a piece, at least: a turn per wave
constexpr int kMaxPieces = 64;        // of a group's keys (the merge weighs them in one wave)
constexpr float kLog2eP = 1.4426950408889634f;
constexpr float kLazyRescale = 8.0f;  // log2 units a block's max may exceed the running max by

__device__ inline uint32_t bf16_pair(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

__device__ inline floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// max and sum over the four lanes that share a query column (l % 16)
__device__ inline float max_rows(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

__device__ inline float sum_rows(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Eight e4m3 bytes (two words) times a power of two, as four words of two bf16.
__device__ inline u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true))};
}

// What the queries of sequence b see.  Hybrid: position p < lc sees [0, p], lc <= p < end sees
// [0, end).  Tree: node r sees [0, lc) and its ancestors among lc .. end - 1.
struct Seq {
    int64_t lc, end, qs;
};

__device__ inline Seq sequence_of(const PagedArgs &a, int b) {
    const int64_t room = static_cast<int64_t>(a.c.max_pages) << a.c.log_page;
    const int64_t lc = max(a.ctx_len[b], 0);
    const int64_t more = a.parent ? a.n_q : 2 * static_cast<int64_t>(a.K) + 3;
    const int64_t end = min(lc + more, room);
    return Seq{min(lc, end), end, a.parent ? lc : static_cast<int64_t>(a.q_start[b])};
}

// Keys [0, kend) that the rows [q0, q1) of a group see, and how they are cut.
struct Cut {
    int64_t kend, chunk;
    int pieces;                // at least 1
};

__device__ inline Cut cut_of(const PagedArgs &a, const Seq &s, int q0, int q1) {
    const int64_t p_lo = s.qs + quot(a.by_grp, q0), p_hi = s.qs + quot(a.by_grp, q1 - 1);
    int64_t kend = s.end;
    if (p_lo >= s.end) kend = 0;                            // all padding: no key
    else if (!a.parent && p_hi < s.lc) kend = max(p_hi + 1, static_cast<int64_t>(0));
    const int64_t part = (kend + a.splits - 1) / a.splits;
    const int64_t chunk = max((part + kStep - 1) / kStep * kStep, static_cast<int64_t>(kMinPiece));
    return Cut{kend, chunk, max(static_cast<int>((kend + chunk - 1) / chunk), 1)};
}

// The sixteen bits from bit `at` (may be negative) of a set of 256.
__device__ inline uint32_t window16(const uint32_t *set, int64_t at) {
    if (at <= -16 || at >= 256) return 0;
    if (at < 0) return (set[0] << -at) & 0xffffu;
    const int w = static_cast<int>(at) >> 5;
    const uint64_t two = set[w] | static_cast<uint64_t>(w < 7 ? set[w + 1] : 0u) << 32;
    return static_cast<uint32_t>(two >> (at & 31)) & 0xffffu;
}

template <int D, bool F8, int RT>
__global__ __launch_bounds__(64 * kWaves, RT == 1 || (F8 && RT == 2) ? 2 : 1) void k_paged_attention(PagedArgs a) {
    constexpr int DS = D / 32;                              // k-steps of the first product
    constexpr int DT = D / 16;                              // d tiles of the second
    constexpr int EB = F8 ? 1 : 2;
    constexpr int KC = D * EB / 64;                         // 16-byte loads of a lane's key
    constexpr int OS = D + 4;                               // floats of a staged row of sums
    __shared__ __attribute__((aligned(16))) float s_o[kWaves][16 * OS];
    __shared__ float2 s_ml[kWaves][16 * RT];
    __shared__ uint32_t s_anc[kMaxSeqRows][8];
    __shared__ int s_up[kMaxSeqRows];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = lane >> 4, l16 = lane & 15;
    const int grp = a.by_grp.d, rows = a.n_q * grp;
    const uint32_t unit = quot(a.by_splits, blockIdx.x);
    const int piece = blockIdx.x - unit * a.by_splits.d;
    const uint32_t bh = quot(a.by_blocks, unit);
    const int blk = unit - bh * a.by_blocks.d;
    const int b = quot(a.by_heads, bh), h = bh - b * a.by_heads.d;
    const int q0 = blk * (16 * RT), q1 = min(q0 + 16 * RT, rows);
    const Seq s = sequence_of(a, b);
    const Cut cut = cut_of(a, s, q0, q1);
    if (piece >= cut.pieces) return;
    const int64_t kbeg = piece * cut.chunk, kend = min(kbeg + cut.chunk, cut.kend);

    if (a.parent) {
        // ancestors of every node, as sets: each round joins the set of the node `up`, twice as
        // far up as the round before
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
            int next = -1;
#pragma unroll
            for (int w = 0; w < 8; ++w) set[w] = up >= 0 ? s_anc[up][w] : 0u;
            if (up >= 0) next = s_up[up];
            __syncthreads();
            if (tid < n) {
#pragma unroll
                for (int w = 0; w < 8; ++w) s_anc[tid][w] |= set[w];
                s_up[tid] = up = next;
            }
        }
        __syncthreads();
    }

    // this lane's query of every row tile.  Keys are taken by a k-step as they lie in memory:
    // bf16 key bytes 64 c + 16 g .. + 15, k-step c; e4m3 the same bytes, k-steps 2c and 2c + 1.
    u32x4 qf[RT][DS];
    int64_t vis[RT];                                        // keys [0, vis) are seen
    int node[RT];
    int64_t vis_min = INT64_MAX;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int qi = q0 + rt * 16 + l16;
        const bool valid = qi < q1;
        const int r = valid ? quot(a.by_grp, qi) : 0;
        const int hq = h * grp + (valid ? qi - r * grp : 0);
        const int64_t p = s.qs + r;
        const bool live = valid && p >= 0 && p < s.end;
        node[rt] = r;
        vis[rt] = !live ? 0 : a.parent || p >= s.lc ? (a.parent ? s.lc : s.end) : p + 1;
        if (live) vis_min = min(vis_min, vis[rt]);
        const char *qrow = static_cast<const char *>(a.q) + ((static_cast<int64_t>(b) * a.n_q + r) * a.Hq + hq) * D * 2;
#pragma unroll
        for (int c = 0; c < DS; ++c) {
            const int d = F8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
            qf[rt][c] = live ? *reinterpret_cast<const u32x4 *>(qrow + d * 2) : u32x4{0, 0, 0, 0};
        }
        if (!live) node[rt] = -1;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) vis_min = min(vis_min, __shfl_xor(vis_min, off));

    floatx4 o[RT][DT];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = -INFINITY;
        l[rt] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[rt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const float sc = a.scale * kLog2eP;

    // A turn's keys lie in up to four pages: of key group l16 / 4 for this lane's key rows, of
    // group g for its values.
    const int32_t *table = a.c.table + static_cast<int64_t>(b) * a.c.max_pages;
    const int P1 = (1 << a.c.log_page) - 1;
    const int kg = l16 >> 2;
    auto ids = [&](int64_t k0, int &idk, int &idv) {
        const int64_t last = a.c.max_pages - 1;
        idk = table[min((k0 + kg * 16) >> a.c.log_page, last)];
        idv = table[min((k0 + g * 16) >> a.c.log_page, last)];
    };
    u32x4 kr[4][KC], vr[DT][EB];
    float ksc = 1.f, vsc = 1.f;
    auto load_keys = [&](int64_t k0, int id) {
        const int64_t pid = max(page_or_none(a.c, id), static_cast<int64_t>(0)), blk_ = pid * a.c.H + h;
        const int place = static_cast<int>(k0 + kg * 16) & P1;
        const char *base = a.c.k + ((blk_ << a.c.log_page) + place + (l16 & 3)) * (D * EB) + g * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < KC; ++c) kr[t][c] = *reinterpret_cast<const u32x4 *>(base + t * 4 * (D * EB) + c * 64);
        if (F8) ksc = a.c.k_scale[blk_];
    };
    auto load_values = [&](int64_t k0, int id) {
        const int64_t pid = max(page_or_none(a.c, id), static_cast<int64_t>(0)), blk_ = pid * a.c.H + h;
        const int place = static_cast<int>(k0 + g * 16) & P1;
        const char *base = a.c.v + ((((blk_ * D) + l16) << a.c.log_page) + place) * EB;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int c = 0; c < EB; ++c)
                vr[t][c] = *reinterpret_cast<const u32x4 *>(base + ((static_cast<int64_t>(t) * 16) << a.c.log_page) * EB + c * 16);
        if (F8) vsc = a.c.v_scale[blk_];
    };

    constexpr int kTurn = kWaves * kStep;
    int64_t k0 = kbeg + wave * kStep;
    int idk, idv, idk1 = 0, idv1 = 0;
    if (k0 < kend) {
        ids(k0, idk, idv);
        ids(k0 + kTurn, idk1, idv1);
        load_keys(k0, idk);
        load_values(k0, idv);
    }
    for (; k0 < kend; k0 += kTurn) {
        const bool more = k0 + kTurn < kend;
        // S^T of the turn
        floatx4 st[RT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u32x4 kf[DS];
#pragma unroll
            for (int c = 0; c < DS; ++c)
                kf[c] = F8 ? widen(kr[t][c / 2][2 * (c % 2)], kr[t][c / 2][2 * (c % 2) + 1], ksc) : kr[t][F8 ? 0 : c];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                st[rt][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DS; ++c) st[rt][t] = mfma(kf[c], qf[rt][c], st[rt][t]);
            }
        }
        const int id_now = idv;
        if (more) {
            load_keys(k0 + kTurn, idk1);
            idv = idv1;
        }
        const int64_t kb = k0 + g * 16;                     // this lane's first key
        const bool none = page_or_none(a.c, id_now) < 0;
        // wave-uniform: a key that some query does not see, or that does not exist
        const bool masked = k0 + kStep > min(vis_min, kend) || __ballot(none) != 0;
        u32x4 pb[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float bm = -INFINITY;
            if (!masked) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        st[rt][t][r] *= sc;
                        bm = fmaxf(bm, st[rt][t][r]);
                    }
            } else {
                const int64_t top = min(vis[rt], kend) - kb;
                uint32_t see = top >= 16 ? 0xffffu : top > 0 ? (1u << top) - 1u : 0u;
                if (a.parent && node[rt] >= 0) {
                    const int64_t real = kend - kb;
                    see |= window16(s_anc[node[rt]], kb - s.lc) & (real >= 16 ? 0xffffu : real > 0 ? (1u << real) - 1u : 0u);
                }
                if (none) see = 0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        st[rt][t][r] = see >> (4 * t + r) & 1 ? st[rt][t][r] * sc : -INFINITY;
                        bm = fmaxf(bm, st[rt][t][r]);
                    }
            }
            bm = max_rows(bm);
            const bool raise = bm > m[rt] + kLazyRescale;   // always when m is still -inf
            if (__builtin_expect(__ballot(raise) != 0, 0)) {
                const float alpha = raise ? __builtin_amdgcn_exp2f(m[rt] - bm) : 1.f;   // 0 from -inf
                if (raise) m[rt] = bm;
                l[rt] *= alpha;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[rt][t] *= alpha;
            }
            // a query that has seen nothing yet keeps m = -inf and adds nothing
            const float mm = m[rt] == -INFINITY ? INFINITY : m[rt];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(st[rt][2 * u + i / 4][i % 4] - mm);
                    l[rt] += p[i];
                }
                pb[rt][u] = u32x4{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3]), bf16_pair(p[4], p[5]), bf16_pair(p[6], p[7])};
            }
        }
        if (masked) {
            // places that hold no key of the sequence may hold anything, as may the scale of a
            // page without one: a weight of zero does not make a NaN harmless
            const int64_t left = none ? 0 : kend - kb;
            const int real = left >= 16 ? 16 : left > 0 ? static_cast<int>(left) : 0;
            if (real == 0) vsc = 1.f;
#pragma unroll
            for (int c = 0; c < EB; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    constexpr int PER = 4 / EB;             // elements of a word
                    const int in = real - (c * 4 + w) * PER;
                    const uint32_t keep = in >= PER ? 0xffffffffu : in > 0 ? (1u << (in * 8 * EB)) - 1u : 0u;
#pragma unroll
                    for (int t = 0; t < DT; ++t) vr[t][c][w] &= keep;
                }
        }
        // O^T += V^T P^T
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4 vf = F8 ? widen(vr[t][0][2 * u], vr[t][0][2 * u + 1], vsc) : vr[t][F8 ? 0 : u];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) o[rt][t] = mfma(vf, pb[rt][u], o[rt][t]);
            }
        if (more) {
            load_values(k0 + kTurn, idv);
            ids(k0 + 2 * kTurn, idk1, idv1);
        }
    }

    // join the waves
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] = sum_rows(l[rt]);
        if (node[rt] < 0) {                                 // no query: unmasked turns weighed its zeros evenly
            m[rt] = -INFINITY;
            l[rt] = 0.f;
        }
        if (g == 0) s_ml[wave][rt * 16 + l16] = make_float2(m[rt], l[rt]);
    }
    __syncthreads();
    const bool whole = cut.pieces == 1;
    const int64_t rows_all = static_cast<int64_t>(a.B) * a.n_q * a.Hq;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_ml[w][rt * 16 + l16].x);
        const float f = m[rt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[rt] - M);
#pragma unroll
        for (int t = 0; t < DT; ++t)
            *reinterpret_cast<floatx4 *>(&s_o[wave][l16 * OS + t * 16 + g * 4]) = o[rt][t] * f;
        __syncthreads();
        // thread: DT components of row tid / 16
        const int row = tid >> 4, d0 = (tid & 15) * DT, qi = q0 + rt * 16 + row;
        float x[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int i = 0; i < DT; ++i) x[i] += s_o[w][row * OS + d0 + i];
        float RM = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) RM = fmaxf(RM, s_ml[w][rt * 16 + row].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float2 ml = s_ml[w][rt * 16 + row];
            L += ml.x == -INFINITY ? 0.f : ml.y * __builtin_amdgcn_exp2f(ml.x - RM);
        }
        if (qi < q1) {
            const int r = quot(a.by_grp, qi);
            const int64_t R = (static_cast<int64_t>(b) * a.n_q + r) * a.Hq + h * grp + (qi - r * grp);
            if (whole) {
                const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;    // NaN stays
                uint32_t w[DT / 2];
#pragma unroll
                for (int i = 0; i < DT / 2; ++i) w[i] = bf16_pair(x[2 * i] * inv, x[2 * i + 1] * inv);
                char *dst = static_cast<char *>(a.out) + (R * D + d0) * 2;
                if constexpr (DT == 8) *reinterpret_cast<u32x4 *>(dst) = u32x4{w[0], w[1], w[2], w[3]};
                else *reinterpret_cast<u32x2 *>(dst) = u32x2{w[0], w[1]};
            } else {
                float *po = a.part_o + (piece * rows_all + R) * D + d0;
#pragma unroll
                for (int i = 0; i < DT; i += 4)
                    __builtin_nontemporal_store(floatx4{x[i], x[i + 1], x[i + 2], x[i + 3]}, reinterpret_cast<floatx4 *>(po + i));
                if ((tid & 15) == 0) a.part_ml[piece * rows_all + R] = make_float2(RM, L);
            }
        }
        __syncthreads();                                    // the staged sums are read
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
    const int grp = a.by_grp.d, tile = 16 * a.row_tiles;
    const int qi = r * grp + hq % grp, q0 = qi / tile * tile;
    const Cut cut = cut_of(a, sequence_of(a, b), q0, min(q0 + tile, a.n_q * grp));
    if (cut.pieces == 1) return;                            // written whole
    const int n = cut.pieces;
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < n) ml = a.part_ml[lane * rows_all + R];
    float M = ml.x;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float l = w * ml.y;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
    const int c = lane % LP, sp = lane / LP;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += SP * U) {
        floatx4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = min(s0 + u * SP + sp, n - 1);
            v[u] = __builtin_nontemporal_load(reinterpret_cast<const floatx4 *>(a.part_o + (s * rows_all + R) * D) + c);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * SP + sp;
            const float ws = __shfl(w, s & 63);
            const bool in = s < n;                          // a clamped piece adds nothing
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[k] = in ? fmaf(ws, v[u][k], acc[k]) : acc[k];
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

template <int D, bool F8>
void run_attention(const PagedArgs &a, unsigned grid, hipStream_t s) {
    const dim3 g(grid), t(64 * kWaves);
    switch (a.row_tiles) {
    case 1: hipLaunchKernelGGL((k_paged_attention<D, F8, 1>), g, t, 0, s, a); break;
    case 2: hipLaunchKernelGGL((k_paged_attention<D, F8, 2>), g, t, 0, s, a); break;
    default: hipLaunchKernelGGL((k_paged_attention<D, F8, 3>), g, t, 0, s, a); break;
    }
}

constexpr int64_t kCus = 256;         // compute units of an MI355X

}  // namespace

PagedPlan paged_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq) {
    PagedPlan p{1, 0, 1, static_cast<int64_t>(B) * n_q * Hq};
    const int64_t tiles = (static_cast<int64_t>(n_q) * (Hq / c.H) + 15) / 16;
    if (B <= 0 || tiles == 0) return p;
    // rows shared out evenly over the fewest workgroups
    const int64_t blocks = (tiles + kMaxRowTiles - 1) / kMaxRowTiles;
    p.row_tiles = static_cast<int32_t>((tiles + blocks - 1) / blocks);
    p.blocks = static_cast<int32_t>((tiles + p.row_tiles - 1) / p.row_tiles);
    const int64_t units = static_cast<int64_t>(B) * c.H * p.blocks;
    const int64_t slots = kCus * (p.row_tiles <= 2 ? 2 : 1);
    const int64_t room = static_cast<int64_t>(c.max_pages) << c.log_page;
    int64_t splits = slots / units;
    splits = splits < (room + kMinPiece - 1) / kMinPiece ? splits : (room + kMinPiece - 1) / kMinPiece;
    p.splits = static_cast<int32_t>(splits < 1 ? 1 : splits > kMaxPieces ? kMaxPieces : splits);
    return p;
}

hipError_t launch_paged_attention(PagedArgs a, const PagedPlan &p, hipStream_t s) {
    const int64_t units = static_cast<int64_t>(a.B) * a.c.H * p.blocks;
    a.row_tiles = p.row_tiles;
    a.splits = p.splits;
    a.by_grp = fast_div(a.Hq / a.c.H);
    a.by_blocks = fast_div(p.blocks);
    a.by_heads = fast_div(a.c.H);
    a.by_splits = fast_div(p.splits);
    a.by_seq_rows = fast_div(static_cast<uint32_t>(a.n_q) * static_cast<uint32_t>(a.Hq));
    a.by_hq = fast_div(a.Hq);
    const unsigned grid = static_cast<unsigned>(units * p.splits);
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
