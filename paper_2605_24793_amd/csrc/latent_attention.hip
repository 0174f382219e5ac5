// Attention over the paged cache of latent vectors, in the absorbed form: all heads' queries meet
// the same vectors, which are keys and values at once.
//
//   s_j = scale (q . c_j + q' . r_j),   o = sum_j softmax(s)_j c_j
//
// One pass over the positions with a running maximum, as in paged_attention.hip.  A sequence's rows (query
// positions x heads) share all of its keys, so a position of 2 (dc + 64) bytes serves 2 (2 dc + 64) operations
// for every row: from about 128 rows on the matrix cores bound it, below the memory.
#include <algorithm>
#include <type_traits>

#include "attend.h"
#include "latent.h"

namespace cospec {
namespace {

constexpr int kKeys = 64;             // of a turn
constexpr int kRotBytes = kRotated * 2;
constexpr int kMinPieceLatent = 256;  // keys of a piece, at least
constexpr float kFar = 60.f;          // log2 units a score may exceed a row's m by (weights and sums are floats)

// 4 bytes per lane into LDS at byte lds + 4 * lane (see load_lds16).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_lds4(const char *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(src) : "memory", "m0");
}
#pragma clang diagnostic pop

// A latent row of the turn holds its sixteen-byte pieces in another order: piece i at place i ^ turned(key), so that
// neither product's reads meet in LDS banks: the first one's, eight rows' same piece, and the second one's,
// which read four rows (bf16) or eight (e4m3) of sixteen components.
template <bool F8> __device__ inline int turned(int key) { return F8 ? key & 7 : (key & 3) << 1 | (key >> 2 & 1); }

// A workgroup takes RT * 32 rows of a sequence, or a piece of its keys, in turns of 64 keys; the next turn's
// latents are on their way into LDS while one is worked on.
//
// The four waves share both products out differently.  Scores: RT = 2, 32 rows and 32 keys each; RT = 1, all
// rows and sixteen keys each.  Sums: all rows and a quarter of the components each, so that a latent is
// read from LDS once or twice for the scores and once for the sums, and a wave holds the queries of 32
// rows and a quarter of the sums.  The rounded weights go from one to the other through LDS.  (With sums of its
// own rows, a wave would hold 256 registers of them beside 144 of queries, and every wave read every latent twice.)
//
// S^T = K Q^T and O^T = C^T P^T: the second product's operand C^T has positions where the rows lie; LDS turns
// them while they are read (ds_read_b64_tr).
//
// A row's weights are 2^(s - m) with m the maximum of the first turn in which it sees a key: that is as exact as with
// the running one, as long as no later score is kFar above it.  Then the sums need not be scaled
// down on the way, and all waves know m.  Where a score is, the piece is taken again: its maxima first, then the
// sums.
template <int DC, bool F8, int RT>
__global__ __launch_bounds__(kThreads, 1) void k_latent_attention(PagedArgs a) {
    constexpr int EB = F8 ? 1 : 2, RB = DC * EB;            // bytes of a latent
    constexpr int ROWS = 32 * RT;
    constexpr int KP = RT == 2 ? 2 : 4;                     // parts of a turn's keys among the waves
    constexpr int QT = RT == 2 ? 1 : 2;                     // query tiles of a wave's scores: 32 wide, or 16
    constexpr int SK = RT == 2 ? 16 : 32;                   // components of a k-step of the first product
    constexpr int CS = DC / SK, RS = kRotated / SK;         // its k-steps, of latents and of rotated keys
    constexpr int NS = RT == 2 ? 16 : 4;                    // scores of a lane and query tile
    constexpr int DT = DC / 4 / 32;                         // component tiles of a wave
    constexpr int kRotAt = kKeys * RB, kScaleAt = kRotAt + kKeys * kRotBytes, kStage = kScaleAt + (F8 ? kKeys * 4 : 0);
    constexpr int RPI = 1024 / RB, PPR = RB / 16;           // rows of a load, pieces of a row
    constexpr int kWeightRow = kKeys * 2 + 16;              // bytes
    __shared__ __attribute__((aligned(128))) char s_ring[2 * kStage];
    __shared__ __attribute__((aligned(16))) char s_weight[ROWS * kWeightRow];
    __shared__ uint32_t s_page[kThreads];
    __shared__ uint32_t s_seen[ROWS][8];                    // ancestors of the rows' nodes
    __shared__ float s_max[KP][ROWS];
    __shared__ float s_sum[KP][ROWS];
    __shared__ uint32_t s_bad[2];                           // of a turn's keys: latent or scale not finite
    __shared__ int s_new, s_far;

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int gh = lane >> 5, l32 = lane & 31;
    const int ql = RT == 2 ? l32 : lane & 15, kg = RT == 2 ? gh : lane >> 4;   // of the first product: query, k-piece
    const int rw = RT == 2 ? wave & 1 : 0, kp = RT == 2 ? wave >> 1 : wave;
    constexpr int TK = kKeys / KP;                          // keys of a wave's scores
    const int rows = a.n_q * a.Hq;
    const Place w_ = place_of(a);
    const int b = w_.b;
    if (b >= a.B) return;
    const int q0 = w_.block * ROWS, q1 = min(q0 + ROWS, rows);
    uint32_t id = a.splits == 1 ? table_entry(a, b, 0) : 0u;
    const int64_t R0 = static_cast<int64_t>(b) * rows;
    u32x4 qf[QT][CS + RS];
    int node[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int qi = min(q0 + rw * 32 + t * 16 + ql, q1 - 1);
        node[t] = quot(a.by_grp, qi);
        const char *qrow = static_cast<const char *>(a.q) + (R0 + qi) * ((DC + kRotated) * 2);
#pragma unroll
        for (int c = 0; c < CS; ++c) {
            // in the order in which the keys' pieces come: of e4m3 a lane's sixteen bytes are two k-steps
            const int d = F8 ? c / 2 * (2 * SK) + kg * 16 + c % 2 * 8 : c * SK + kg * 8;
            qf[t][c] = *reinterpret_cast<const u32x4 *>(qrow + d * 2);
        }
#pragma unroll
        for (int c = 0; c < RS; ++c) qf[t][CS + c] = *reinterpret_cast<const u32x4 *>(qrow + (DC + c * SK + kg * 8) * 2);
    }
    const Seq s = sequence_of(a, b);
    const Cut cut = cut_of(a, s, q0, q1);
    if (w_.piece >= cut.pieces) return;
    const int kbeg = w_.piece * cut.chunk, kend = min(kbeg + cut.chunk, cut.kend);
    const int all_see = seen_by_all(a, s, q0, kend);        // keys below are seen by every row that sees any

    const int P1 = (1 << a.c.log_page) - 1;
    int first_page = 0, last_page = 0;                      // of those in LDS
    bool any_none = false;
    const uint32_t ring = uniform(lds_address(s_ring));
    auto page_of = [&](int key) { return s_page[min(key >> a.c.log_page, last_page) - first_page]; };
    // this wave's sixteen keys of a turn (all of one page), into LDS
    auto load = [&](int k0, uint32_t stage) {
        const int key = k0 + wave * 16;
        const int64_t page = uniform(page_of(key) & ~kNone);
        const int64_t place = (page << a.c.log_page) + (key & P1);
        const char *c = a.c.k + place * RB, *rot = a.c.v + place * kRotBytes;
        const uint32_t at = stage + wave * (16 * RB);
#pragma unroll
        for (int i = 0; i < 16 / RPI; ++i) {
            const int row = i * RPI + lane / PPR;
            load_lds16<false>(c + row * RB + ((lane % PPR) ^ turned<F8>(row)) * 16, at + i * 1024);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = i * 8 + lane / 8;
            load_lds16<false>(rot + row * kRotBytes + ((lane % 8) ^ (row & 7)) * 16, stage + kRotAt + wave * (16 * kRotBytes) + i * 1024);
        }
        if (F8 && wave == 0) {
            const int mine = k0 + lane;
            const int64_t p = page_of(mine) & ~kNone;
            load_lds4(reinterpret_cast<const char *>(a.c.k_scale + (p << a.c.log_page) + (mine & P1)), stage + kScaleAt);
        }
    };
    auto look_up = [&](int from, int to, uint32_t entry) {  // of keys [from, to), this thread's table entry given
        first_page = from >> a.c.log_page;
        last_page = (to - 1) >> a.c.log_page;
        const bool in = tid <= last_page - first_page, none = entry >= static_cast<uint32_t>(a.c.n_pages);
        if (in) s_page[tid] = none ? kNone : entry;         // a page that is none is read as page 0, and not used
        any_none = __syncthreads_or(in && none);
    };
    if (a.parent) {
        uint32_t(*const anc)[8] = reinterpret_cast<uint32_t(*)[8]>(s_ring);
        find_ancestors(a, b, anc, reinterpret_cast<int *>(s_ring + kMaxSeqRows * 32));
        for (int i = tid; i < ROWS * 8; i += kThreads) s_seen[i / 8][i % 8] = anc[quot(a.by_grp, min(q0 + i / 8, q1 - 1))][i % 8];
        __syncthreads();
    }

    // scores are taken as |scale| (+-q) . k, so that the largest product is the largest score
    int vis[QT];                                            // keys [0, vis) are seen
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int64_t p = s.qs + node[t];
        const bool live = q0 + rw * 32 + t * 16 + ql < q1 && p >= 0 && p < s.end;
        vis[t] = !live ? 0 : a.parent ? s.lc : p >= s.lc ? s.end : static_cast<int>(p) + 1;
        if (!live) node[t] = -1;
#pragma unroll
        for (int c = 0; c < CS + RS; ++c)
#pragma unroll
            for (int x = 0; x < 4; ++x) qf[t][c][x] = live ? qf[t][c][x] ^ flip : 0u;
    }
    const float sc = fmaxf(fabsf(a.scale) * kLog2eP, 1.17549435e-38f);

    floatx16 o[RT][DT];
    float m[QT], l[QT];                                     // l: of this lane's keys alone
    auto begin = [&] {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][dt][i] = 0.f;
#pragma unroll
        for (int t = 0; t < QT; ++t) l[t] = 0.f;
    };
    begin();
#pragma unroll
    for (int t = 0; t < QT; ++t) m[t] = -INFINITY;
    if (tid == 0) s_new = s_far = 0;

    // where this lane reads: keys' pieces, rotated keys' pieces, latents' components, weights
    const int krow = kp * TK + ql;
    const uint32_t k_at = krow * RB + ((kg ^ turned<F8>(ql)) & 7) * 16;
    const uint32_t r_at = kRotAt + krow * kRotBytes + ((kg ^ ql) & 7) * 16;
    uint32_t v_at;
    {
        const int j = lane & 15, cg = lane >> 4 & 1, row = 8 * gh + (F8 ? j >> 1 : j >> 2);
        const int piece = wave * (PPR / 4) + (F8 ? cg : 2 * cg + (j >> 1 & 1));
        v_at = row * RB + (piece >> 3) * 128 + ((piece ^ turned<F8>(row)) & 7) * 16 + (j & 1) * 8;
    }
    const char *const w_at = s_weight + l32 * kWeightRow + gh * 16;

    const int segment = kSegment << a.c.log_page;
    // finding: only the rows' maxima, into m
    auto pass = [&](bool finding) {
        for (int seg = kbeg; seg < kend; seg += segment) {
            const int seg_end = min(seg + segment, kend);
            if (seg > kbeg || a.splits > 1) id = table_entry(a, b, seg >> a.c.log_page);
            if (seg > kbeg) __syncthreads();                // the pages of the segment before are used up
            look_up(seg, seg_end, id);
            load(seg, ring);
            for (int k0 = seg, buf = 0; k0 < seg_end; k0 += kKeys, buf ^= 1) {
                wait_vm<0>();                               // this wave's part of the turn
                lds_barrier();                              // ... and the others'; the turn before is used up
                if (k0 + kKeys < seg_end) load(k0 + kKeys, ring + (buf ^ 1) * kStage);
                char *const stage = s_ring + buf * kStage;
                const bool masked = k0 + kKeys > all_see || any_none;   // the same in the whole workgroup
                if (masked) {
                    // Places that hold no key of the sequence may hold anything, and a weight of zero does not make
                    // a NaN harmless: they become zeros, as do latents that are not finite, whose keys are marked.
                    if (tid < 2) s_bad[tid] = 0;
                    lds_barrier();
                    const int key = tid >> 2, part = tid & 3;
                    const bool real = k0 + key < kend && page_of(k0 + key) < kNone;
                    float *const scale = reinterpret_cast<float *>(stage + kScaleAt) + key;
                    uint32_t top = 0;
#pragma unroll 2
                    for (int i = 0; i < PPR / 4; ++i) {
                        u32x4 *at = reinterpret_cast<u32x4 *>(stage + key * RB + (part + 4 * i) * 16);
                        u32x4 x = *at;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t t = not_finite<F8>(x[e], 0x01010101u);
                            top |= t;
                            x[e] = real ? x[e] & ~(t | (t - (t >> (F8 ? 7 : 15)))) : 0u;
                        }
                        *at = x;
                    }
                    bool bad = top != 0;
                    if constexpr (F8) {
                        const float sv = *scale;
                        const bool wild = !(fabsf(sv) < INFINITY);
                        bad |= wild;
                        wait_lds();
                        if (part == 0 && (wild || !real)) *scale = 0.f;   // (the four of a key are of one wave)
                    }
                    if (real && bad) atomicOr(&s_bad[key >> 5], 1u << (key & 31));
                    lds_barrier();
                }
                // S^T
                typedef std::conditional_t<RT == 2, floatx16, floatx4> Tile;
                Tile st[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < NS; ++i) st[t][i] = 0.f;
                auto multiply = [&](u32x4 k, int c) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        if constexpr (RT == 2) st[t] = mfma32(k, qf[t][c], st[t]);
                        else st[t] = mfma(k, qf[t][c], st[t]);
                    }
                };
                // sixteen-byte pieces of a key that a load's lanes take side by side
                constexpr int LP = RT == 2 ? 2 : 4, PER = 8 / LP;
                constexpr int LOADS = CS / (F8 ? 2 : 1);
#pragma unroll
                for (int c = 0; c < LOADS; ++c) {
                    const u32x4 raw = *reinterpret_cast<const u32x4 *>(stage + (k_at ^ (c % PER * LP * 16)) + c / PER * 128);
                    if constexpr (F8) {
                        multiply(widen(raw[0], raw[1], 1.f), 2 * c);
                        multiply(widen(raw[2], raw[3], 1.f), 2 * c + 1);
                    } else {
                        multiply(raw, c);
                    }
                }
                float sv[F8 ? NS : 1];                      // scales of this lane's keys
                if constexpr (F8) {
#pragma unroll
                    for (int e = 0; e < NS / 4; ++e) {
                        const floatx4 x = *reinterpret_cast<const floatx4 *>(stage + kScaleAt + (kp * TK + 8 * e + 4 * kg) * 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) sv[4 * e + i] = x[i];
                    }
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int i = 0; i < NS; ++i) st[t][i] *= sv[i];
                }
#pragma unroll
                for (int c = 0; c < RS; ++c)
                    multiply(*reinterpret_cast<const u32x4 *>(stage + (r_at ^ (c * LP * 16))), CS + c);
                if (masked) {
                    const int kb = k0 + kp * TK;
                    uint32_t real = low_bits(kend - kb);
                    if (page_of(kb) >= kNone) real &= 0xffff0000u;
                    if (TK == 32 && page_of(kb + 16) >= kNone) real &= 0x0000ffffu;
                    const uint32_t bad = s_bad[kp * TK / 32] >> (kp * TK % 32 + 4 * kg);
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        uint32_t see = low_bits(vis[t] - kb);
                        if (a.parent && node[t] >= 0) see |= window32(s_seen[rw * 32 + t * 16 + ql], kb - s.lc);
                        see = (see & real) >> (4 * kg);
#pragma unroll
                        for (int i = 0; i < NS; ++i) {
                            const int bit = 8 * (i / 4) + i % 4;
                            if (!(see >> bit & 1)) st[t][i] = -INFINITY;
                            else if (bad >> bit & 1) st[t][i] = NAN;
                        }
                    }
                }
                float bm[QT];
                bool fresh = false;                         // a row's first keys, or a score far above m
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    bm[t] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < NS; ++i) bm[t] = fmaxf(bm[t], st[t][i]);
                    if constexpr (RT == 2) {
                        const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(bm[t]), __float_as_uint(bm[t]), false, false);
                        bm[t] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
                    } else {
                        bm[t] = max_rows(bm[t]);
                    }
                    bm[t] *= sc;
                    fresh |= bm[t] > m[t] + kFar;           // always when m is still -inf
                }
                if (finding) {
#pragma unroll
                    for (int t = 0; t < QT; ++t) m[t] = fmaxf(m[t], bm[t]);
                    continue;
                }
                float sum[QT];
                auto weigh = [&] {
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        // a query that has seen nothing yet keeps m = -inf and adds nothing
                        const float mm = m[t] == -INFINITY ? INFINITY : m[t];
                        sum[t] = 0.f;
                        char *to = s_weight + (rw * 32 + t * 16 + ql) * kWeightRow + (kp * TK + 4 * kg) * 2;
#pragma unroll
                        for (int e = 0; e < NS / 4; ++e) {
                            float p[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                p[i] = __builtin_amdgcn_exp2f(fmaf(st[t][4 * e + i], sc, -mm));
                                sum[t] += p[i];
                                if constexpr (F8) p[i] *= sv[4 * e + i];
                            }
                            *reinterpret_cast<u32x2 *>(to + e * 16) = u32x2{bf16_pair(p[0], p[1]), bf16_pair(p[2], p[3])};
                        }
                    }
                };
                weigh();
                if (__ballot(fresh) != 0 && lane == 0) s_new = 1;
                lds_barrier();                              // the weights are there
                if (__builtin_expect(uniform(s_new), 0)) {
                    // the same maximum in all waves, then the weights again
                    if (kg == 0) {
#pragma unroll
                        for (int t = 0; t < QT; ++t) s_max[kp][rw * 32 + t * 16 + ql] = bm[t];
                    }
                    lds_barrier();
                    if (tid == 0) s_new = 0;
                    bool far = false;
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        float top = -INFINITY;
#pragma unroll
                        for (int i = 0; i < KP; ++i) top = fmaxf(top, s_max[i][rw * 32 + t * 16 + ql]);
                        if (m[t] == -INFINITY) m[t] = top;
                        else far |= top > m[t] + kFar;
                    }
                    if (__ballot(far) != 0 && lane == 0) s_far = 1;
                    weigh();
                    lds_barrier();
                    if (uniform(s_far)) return;
                }
#pragma unroll
                for (int t = 0; t < QT; ++t) l[t] += sum[t];
                // O^T += C^T P^T
#pragma unroll
                for (int v = 0; v < kKeys / 16; ++v) {
                    u32x4 pb[RT];
#pragma unroll
                    for (int t = 0; t < RT; ++t) pb[t] = *reinterpret_cast<const u32x4 *>(w_at + t * (32 * kWeightRow) + v * 32);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        u32x4 vf;
                        const char *at = stage + v * 16 * RB;
                        if constexpr (F8) {
                            const i32x2 raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(at + (v_at ^ (dt % 4 * 32))));
                            vf = widen(raw[0], raw[1], 1.f);
                        } else {
                            const uint32_t here = (v_at ^ (dt % 2 * 64)) + dt / 2 * 128;
                            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + here)));
                            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * RB + (here ^ 16))));
                            vf = u32x4{lo[0], lo[1], hi[0], hi[1]};
                        }
#pragma unroll
                        for (int t = 0; t < RT; ++t) o[t][dt] = mfma32(vf, pb[t], o[t][dt]);
                    }
                }
            }
        }
    };
    // every row's maximum and sum, joined over the parts of the keys
    auto join_max = [&] {
        __syncthreads();
        if (kg == 0) {
#pragma unroll
            for (int t = 0; t < QT; ++t) s_max[kp][rw * 32 + t * 16 + ql] = m[t];
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int i = 0; i < KP; ++i) m[t] = fmaxf(m[t], s_max[i][rw * 32 + t * 16 + ql]);
        }
    };
    pass(false);
    __syncthreads();
    if (__builtin_expect(uniform(s_far), 0)) {
        wait_vm<0>();                                       // (a turn may still be on its way)
        __syncthreads();
        if (tid == 0) s_new = s_far = 0;
        pass(true);
        join_max();
        begin();
        pass(false);
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        if constexpr (RT == 1) l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
        if (kg == 0) {
            s_sum[kp][rw * 32 + t * 16 + ql] = node[t] >= 0 ? l[t] : 0.f;   // (unmasked turns give padding rows some weights)
            s_max[kp][rw * 32 + t * 16 + ql] = node[t] >= 0 ? m[t] : -INFINITY;
        }
    }
    __syncthreads();
    // O^T tile dt, elements 4e .. 4e + 3: components 32 dt + 8 e + 4 gh + 0..3 of the wave's quarter, of row l32
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = t * 32 + l32, qi = q0 + row;
        if (qi >= q1) continue;
        float L = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i) L += s_sum[i][row];
        if (cut.pieces == 1) {
            const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;   // NaN stays
            char *dst = static_cast<char *>(a.out) + ((R0 + qi) * DC + wave * (DC / 4) + 4 * gh) * 2;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    floatx4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = L == 0.f ? 0.f : o[t][dt][4 * e + i] * inv;
                    *reinterpret_cast<u32x2 *>(dst + (32 * dt + 8 * e) * 2) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
                }
        } else {
            const int64_t at = w_.piece * (static_cast<int64_t>(a.B) * rows) + R0 + qi;
            float *po = a.part_o + at * DC + wave * (DC / 4) + 4 * gh;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<floatx4 *>(po + 32 * dt + 8 * e) =
                        floatx4{o[t][dt][4 * e], o[t][dt][4 * e + 1], o[t][dt][4 * e + 2], o[t][dt][4 * e + 3]};
            if (wave == 0 && gh == 0) a.part_ml[at] = make_float2(s_max[0][row], L);
        }
    }
}

// Joins the pieces of the rows that were cut: one wave per row, lane s weighs piece s, then each lane
// takes DC / 64 components of every piece.
template <int DC>
__global__ __launch_bounds__(256) void k_latent_join(PagedArgs a) {
    constexpr int EACH = DC / 256;                          // four components at a time
    const int lane = threadIdx.x & 63;
    const int64_t rows_all = static_cast<int64_t>(a.B) * a.n_q * a.Hq;
    const int64_t R = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (R >= rows_all) return;
    const int rows = a.n_q * a.Hq;
    const int b = quot(a.by_seq_rows, static_cast<uint32_t>(R));
    const int qi = static_cast<int>(R - static_cast<int64_t>(b) * rows);
    const int tile = 32 * a.row_waves, q0 = qi / tile * tile;
    float2 ml = a.part_ml[min(lane, a.splits - 1) * rows_all + R];
    const Cut cut = cut_of(a, sequence_of(a, b), q0, min(q0 + tile, rows));
    if (cut.pieces == 1) return;                            // written whole
    const int n = cut.pieces;
    if (lane >= n) ml = make_float2(-INFINITY, 0.f);
    float M = ml.x;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float l = ml.x == -INFINITY ? 0.f : w * ml.y;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
    floatx4 acc[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) acc[e] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < n; ++p) {
        const float wp = __shfl(w, p);
        const bool none = __shfl(ml.x, p) == -INFINITY;     // (its sums may be anything)
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const floatx4 v = *(reinterpret_cast<const floatx4 *>(a.part_o + (p * rows_all + R) * DC) + e * 64 + lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[e][i] = none ? acc[e][i] : fmaf(wp, v[i], acc[e][i]);
        }
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        *(reinterpret_cast<u32x2 *>(static_cast<char *>(a.out) + R * DC * 2) + e * 64 + lane) =
            u32x2{bf16_pair(acc[e][0] * inv, acc[e][1] * inv), bf16_pair(acc[e][2] * inv, acc[e][3] * inv)};
}

template <int DC, bool F8> void run_attention(const PagedArgs &a, unsigned grid, hipStream_t s) {
    if (a.row_waves == 2) hipLaunchKernelGGL((k_latent_attention<DC, F8, 2>), dim3(grid), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_latent_attention<DC, F8, 1>), dim3(grid), dim3(kThreads), 0, s, a);
}

}  // namespace

PagedPlan latent_plan(const PageArgs &c, int32_t B, int32_t n_q, int32_t Hq) {
    PagedPlan p{1, 1, 0, 1, kMinPieceLatent, static_cast<int64_t>(B) * n_q * Hq, 0};
    const int64_t rows = static_cast<int64_t>(n_q) * Hq;
    if (B <= 0 || rows == 0) return p;
    p.row_waves = rows <= 32 ? 1 : 2;
    p.blocks = static_cast<int32_t>((rows + 32 * p.row_waves - 1) / (32 * p.row_waves));
    const int64_t units = static_cast<int64_t>(B) * p.blocks, room = static_cast<int64_t>(c.max_pages) << c.log_page;
    // a workgroup fills a CU: as many pieces as give each one
    if (units <= kCus / 2)
        p.splits = static_cast<int32_t>(std::max<int64_t>(
            std::min({kCus / units, (room + p.min_piece - 1) / p.min_piece, kMaxPieces}), 1));
    p.grid = (static_cast<int64_t>(B) * p.splits + kXcds - 1) / kXcds * kXcds * p.blocks;     // each XCD takes as many
    return p;
}

hipError_t launch_latent_attention(PagedArgs a, const PagedPlan &p, hipStream_t s) {
    a.row_tiles = p.row_tiles;
    a.row_waves = p.row_waves;
    a.splits = p.splits;
    a.min_piece = p.min_piece;
    a.by_grp = fast_div(a.Hq);
    a.by_blocks = fast_div(p.blocks);
    a.by_heads = fast_div(1);
    a.by_splits = fast_div(p.splits);
    a.by_seq_rows = fast_div(static_cast<uint32_t>(a.n_q) * static_cast<uint32_t>(a.Hq));
    a.by_hq = fast_div(a.Hq);
    const unsigned grid = static_cast<unsigned>(p.grid);
    if (a.c.D == 512) a.c.f8 ? run_attention<512, true>(a, grid, s) : run_attention<512, false>(a, grid, s);
    else a.c.f8 ? run_attention<256, true>(a, grid, s) : run_attention<256, false>(a, grid, s);
    if (p.splits > 1) {
        const dim3 jgrid(static_cast<unsigned>((p.rows + 3) / 4));
        if (a.c.D == 512) hipLaunchKernelGGL(k_latent_join<512>, jgrid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL(k_latent_join<256>, jgrid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace cospec
