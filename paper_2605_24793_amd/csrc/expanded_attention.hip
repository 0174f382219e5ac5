// The latent cache's attention in the expanded form: every head has keys and values of its own beside
// the rotated key that all heads share, for whole inputs, not paged.
//
// One pass over the keys with a running maximum, as in paged_attention.hip.  A workgroup takes 128 rows of one
// head and sequence, 32 a wave, and its waves share the keys, in turns of 64 that are on their way into LDS
// while the turn before is worked on.  Two workgroups share a CU (their turns fill its LDS to the last byte): while one
// finds weights, the other one multiplies; one of 256 rows, whose waves do the same at the same time, took 233 us where
// two take 200 (4 x 2065 rows, 32 heads, 128 components), and left more rows empty.
//
// S^T = K Q^T and O^T = V^T P^T with 32 x 32 products: a lane holds query l % 32 and the keys 8 (i / 4) +
// 4 (l / 32) + i % 4 of a tile, whose rounded weights are the second product's operand as they
// stand; the values are turned while they are read from LDS (ds_read_b64_tr).
#include <algorithm>

#include "attend.h"
#include "latent.h"

namespace cospec {
namespace {

constexpr int kKeys = 64;             // of a turn
constexpr int kWavesExpanded = 4;     // of a workgroup

// Heads that an XCD works on at a time.  With one, its workgroups read the same rows from its L2 at the same time, but those of
// one head lie in few of the L2's channels, and the longest rows come late.  4 x 2065 rows of 32 heads, 128 components:
// 1 head 213 us, 4 heads 202, 8 heads 198, 16 heads 198.
constexpr int64_t kHeadsTogether = 8;

// Row `key` of a turn holds its sixteen-byte pieces at place i ^ turned(key), so that sixteen rows' same piece, and four
// rows' four pieces, lie in different ones of the 64 banks; rotated keys, of which a row reaches over 32 banks, likewise.
template <int D> __device__ inline int turned(int key) {
    return D == 128 ? (key & 3) << 2 | (key >> 2 & 3) : (key >> 1 & 1) << 2 | (key >> 2 & 3);
}

__device__ inline int turned_rotated(int key) { return key >> 1 & 7; }

template <int D>
__global__ __launch_bounds__(64 * kWavesExpanded, 2) void k_expanded_attention(ExpandedArgs a) {
    constexpr int NW = kWavesExpanded, RB = D * 2, DR = kRotated;
    constexpr int CS = D / 16, RS = DR / 16, DT = D / 32, KT = kKeys / 32;
    constexpr int kRotAt = kKeys * RB, kValuesAt = kRotAt + kKeys * DR * 2, kStage = kValuesAt + kKeys * RB;
    constexpr int PPR = RB / 16;                            // pieces of a row
    constexpr int ROWS = 32 * NW;
    __shared__ __attribute__((aligned(256))) char s_ring[2 * kStage];

    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int gh = lane >> 5, l32 = lane & 31;
    // An XCD takes consecutive heads, `together` of them at a time: the last rows of each first, which see the most keys.
    const uint32_t slot = blockIdx.x / kXcds, x = quot(a.by_together, slot), group = quot(a.by_blocks, x);
    const int block = a.by_blocks.d - 1 - (x - group * a.by_blocks.d);
    const uint32_t mine = group * a.by_together.d + (slot - x * a.by_together.d), bh = blockIdx.x % kXcds * a.heads_each + mine;
    if (mine >= static_cast<uint32_t>(a.heads_each)) return;
    const int b = quot(a.by_heads, bh), h = static_cast<int>(bh - b * a.by_heads.d);
    if (b >= a.B) return;
    const int q0 = block * ROWS, q1 = min(q0 + ROWS, a.n_q);
    const int qi = q0 + wave * 32 + l32;
    const bool valid = qi < q1;
    const int64_t R = (static_cast<int64_t>(b) * a.n_q + min(qi, q1 - 1)) * a.H + h;
    const char *qrow = a.q + R * ((D + DR) * 2);
    u32x4 qf[CS + RS];
#pragma unroll
    for (int c = 0; c < CS + RS; ++c) qf[c] = *reinterpret_cast<const u32x4 *>(qrow + (c * 16 + gh * 8) * 2);
    const int64_t lc0 = max(scalar_load(a.ctx_len + b), 0);
    const int end = static_cast<int>(min(lc0 + 2 * static_cast<int64_t>(a.K) + 3, static_cast<int64_t>(a.L)));
    const int lc = static_cast<int>(min(lc0, static_cast<int64_t>(end)));
    const int64_t qs = scalar_load(a.q_start + b);
    // keys [0, kend) that some row sees, [0, all_see) that every row sees that sees any
    const int64_t p_lo = qs + q0, p_hi = qs + q1 - 1;
    int kend = p_lo >= end ? 0 : p_hi < lc ? max(static_cast<int>(p_hi) + 1, 0) : end;
    const int64_t p_first = max(p_lo, static_cast<int64_t>(0));
    const int all_see = p_first >= lc ? kend : min(static_cast<int>(p_first) + 1, kend);

    const int64_t p_q = qs + qi;
    const bool live = valid && p_q >= 0 && p_q < end;
    const int vis = !live ? 0 : p_q >= lc ? end : static_cast<int>(p_q) + 1;
    int most = vis;                                         // of the wave's rows
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) most = max(most, __shfl_xor(most, off));
    most = uniform(most);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int c = 0; c < CS + RS; ++c)
#pragma unroll
        for (int x = 0; x < 4; ++x) qf[c][x] = live ? qf[c][x] ^ flip : 0u;
    const float sc = fmaxf(fabsf(a.scale) * kLog2eP, 1.17549435e-38f);

    const uint32_t ring = uniform(lds_address(s_ring));
    const char *const kb = a.k + (static_cast<int64_t>(b) * a.L * a.ld_k + h * a.head_k) * 2;
    const char *const vb = a.v + (static_cast<int64_t>(b) * a.L * a.ld_v + h * a.head_v) * 2;
    const char *const rb = a.k_r + static_cast<int64_t>(b) * a.L * a.ld_r * 2;
    // A turn's keys, values and rotated keys.  The lanes' offsets are made once; the last turn's loads, which read keys
    // past the last one as the last one, and those of unusual strides make addresses of their own.
    constexpr int NI = kKeys * RB / 1024 / NW, NR = kKeys * DR * 2 / 1024 / NW;   // a wave's loads of keys (values), of rotated keys
    constexpr int RPI = 1024 / RB;                          // keys of a load
    uint32_t k_off[NI], v_off[NI], r_off[NR];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int row = (wave * NI + i) * RPI + lane / PPR, piece = (lane % PPR) ^ turned<D>(row);
        k_off[i] = static_cast<uint32_t>(row * a.ld_k * 2) + piece * 16 - i * 1024;
        v_off[i] = static_cast<uint32_t>(row * a.ld_v * 2) + piece * 16 - i * 1024;
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int row = (wave * NR + i) * 8 + lane / 8;
        r_off[i] = static_cast<uint32_t>(row * a.ld_r * 2) + ((lane % 8) ^ turned_rotated(row)) * 16 - i * 1024;
    }
    const bool usual = min(a.ld_k, a.ld_v) >= D && max(max(a.ld_k, a.ld_v), a.ld_r) <= 1 << 23;   // offsets of 32 bits, none negative
    const int whole = usual ? kend : 0;                     // turns that end by here are loaded so
    auto load_part = [&](int part, int64_t key, uint32_t stage) __attribute__((always_inline)) {
        if (part == 0) load_lds_rows<NI>(kb + key * a.ld_k * 2, k_off, stage + wave * (NI * 1024));
        else if (part == 1) load_lds_rows<NI>(vb + key * a.ld_v * 2, v_off, stage + kValuesAt + wave * (NI * 1024));
        else load_lds_rows<NR>(rb + key * a.ld_r * 2, r_off, stage + kRotAt + wave * (NR * 1024));
    };
    auto load = [&](int k0, uint32_t stage) {
        if (k0 + kKeys <= whole) {
#pragma unroll
            for (int part = 0; part < 3; ++part) load_part(part, k0, stage);
        } else {
            int at = lane;
            asm volatile("" : "+v"(at));                    // (its addresses are not kept)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int row = (wave * NI + i) * RPI + at / PPR, piece = (at % PPR) ^ turned<D>(row);
                const int64_t key = min(k0 + row, kend - 1);
                load_lds16<false>(kb + key * a.ld_k * 2 + piece * 16, stage + (wave * NI + i) * 1024);
                load_lds16<false>(vb + key * a.ld_v * 2 + piece * 16, stage + kValuesAt + (wave * NI + i) * 1024);
            }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int row = (wave * NR + i) * 8 + at / 8;
                const int64_t key = min(k0 + row, kend - 1);
                load_lds16<false>(rb + key * a.ld_r * 2 + ((at % 8) ^ turned_rotated(row)) * 16, stage + kRotAt + (wave * NR + i) * 1024);
            }
        }
    };

    floatx16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m = -INFINITY, l = 0.f;                           // l: of this lane's keys alone
    const uint32_t k_at = l32 * RB + (gh ^ turned<D>(l32)) * 16;
    const uint32_t r_at = kRotAt + l32 * (DR * 2) + (gh ^ turned_rotated(l32)) * 16;
    const int vj = lane & 15, vrow = 4 * gh + (vj >> 2);
    const uint32_t v_at = kValuesAt + vrow * RB + ((2 * (lane >> 4 & 1) + (vj >> 1 & 1)) ^ turned<D>(vrow)) * 16 + (vj & 1) * 8;

    if (kend > 0) load(0, ring);
    for (int k0 = 0, buf = 0; k0 < kend; k0 += kKeys, buf ^= 1) {
        wait_vm<0>();                                       // this wave's part of the turn
        lds_barrier();                                      // ... and the others'; the turn before is used up
        // The next turn's loads go out between this one's products where their addresses are ready: ten loads of a wave take
        // 650 cycles to go out when all waves of the CU load at once (201 us all in front, 192 between).
        const uint32_t next = ring + (buf ^ 1) * kStage;
        const bool between = k0 < most && k0 + 2 * kKeys <= whole;
        if (!between && k0 + kKeys < kend) load(k0 + kKeys, next);
        char *const stage = s_ring + buf * kStage;
        const bool masked = k0 + kKeys > all_see;           // the same in the whole workgroup
        if (masked) {
            // values that are not finite become zeros (a weight of zero would not keep them from the rows that
            // do not see them), and their rotated keys NaN: so are the scores then of the rows that do
            constexpr int PT = NW;                          // threads of a key
            const int key = tid / PT;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < (PPR + PT - 1) / PT; ++i) {
                const int piece = tid % PT + PT * i;
                u32x4 *at = reinterpret_cast<u32x4 *>(stage + kValuesAt + key * RB + piece * 16);
                u32x4 x = *at;
                uint32_t any = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t t = not_finite<false>(x[e], 0u);
                    any |= t;
                    x[e] &= ~(t | (t - (t >> 15)));
                }
                if (any) *at = x;
                top |= any;
            }
            if (top) *reinterpret_cast<uint32_t *>(stage + kRotAt + key * (DR * 2)) = 0x7fff7fffu;
            lds_barrier();
        }
        if (k0 < most) {
            floatx16 st[KT];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) st[t][i] = 0.f;
            // operands are read from LDS a group ahead of the products that take them
            constexpr int G = 2, NG = (CS + RS) / G;
            u32x4 kf[2][G][KT];
            auto read_keys = [&](int g) __attribute__((always_inline)) {
#pragma unroll
                for (int x = 0; x < G; ++x)
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        const int c = g * G + x;
                        kf[g & 1][x][t] = c < CS ? *reinterpret_cast<const u32x4 *>(stage + t * (32 * RB) + (k_at ^ (c * 32)))
                                                 : *reinterpret_cast<const u32x4 *>(stage + t * (32 * DR * 2) + (r_at ^ ((c - CS) * 32)));
                    }
            };
            u32x4 vf[2][DT];
            auto read_values = [&](int v) __attribute__((always_inline)) {
                const char *const rows = stage + v * 16 * RB;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const uint32_t at = v_at ^ (dt * 64);
                    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(rows + at)));
                    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(rows + 8 * RB + (at ^ 32))));
                    vf[v & 1][dt] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                }
            };
            read_keys(0);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                if (g + 1 < NG) read_keys(g + 1);
                else read_values(0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < G; ++x)
#pragma unroll
                    for (int t = 0; t < KT; ++t) st[t] = mfma32(kf[g & 1][x][t], qf[g * G + x], st[t]);
                __builtin_amdgcn_sched_barrier(0);
                if (g < 3 && between) load_part(g, k0 + kKeys, next);
            }
            if (masked) {
#pragma unroll
                for (int t = 0; t < KT; ++t) {
                    const uint32_t see = low_bits(vis - (k0 + 32 * t)) >> (4 * gh);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int bit = 8 * (i / 4) + i % 4;
                        if (!(see >> bit & 1)) st[t][i] = -INFINITY;
                    }
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
                l *= alpha;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[t][i] *= alpha;
            }
            // a query that has seen nothing yet keeps m = -inf and adds nothing
            const float mm = m == -INFINITY ? INFINITY : m;
            u32x4 pb[KT][2];
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int e = 8 * v + 2 * i;
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(st[t][e], sc, -mm)), p1 = __builtin_amdgcn_exp2f(fmaf(st[t][e + 1], sc, -mm));
                        l += p0 + p1;
                        pb[t][v][i] = bf16_pair(p0, p1);
                    }
#pragma unroll
            for (int v = 0; v < 2 * KT; ++v) {
                if (v + 1 < 2 * KT) read_values(v + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = mfma32(vf[v & 1][dt], pb[v / 2][v & 1], o[dt]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    l += __shfl_xor(l, 32);
    if (!valid) return;
    // O^T tile t, elements 4e .. 4e + 3: components 32 t + 8 e + 4 gh + 0..3 of this lane's row
    // A row that sees nothing gets zeros (unmasked turns gave it some weights).  NaN stays, also in sums without a weight, as
    // scores of minus infinity alone leave them where a value is not finite.
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    char *dst = a.out + (R * D + 4 * gh) * 2;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            floatx4 x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = live ? o[t][4 * e + i] * inv : 0.f;
            *reinterpret_cast<u32x2 *>(dst + (32 * t + 8 * e) * 2) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
        }
}

constexpr int kRowsExpanded = 32 * kWavesExpanded;

int64_t row_blocks(int32_t n_q) { return (static_cast<int64_t>(n_q) + kRowsExpanded - 1) / kRowsExpanded; }

}  // namespace

int64_t heads_each(int32_t B, int32_t H) { return (static_cast<int64_t>(B) * H + kXcds - 1) / kXcds; }

int64_t expanded_workgroups(int32_t B, int32_t n_q, int32_t H) {
    const int64_t each = heads_each(B, H), together = std::max<int64_t>(std::min(each, kHeadsTogether), 1);
    return kXcds * ((each + together - 1) / together * together) * row_blocks(n_q);
}

hipError_t launch_expanded_attention(ExpandedArgs a, hipStream_t s) {
    a.heads_each = static_cast<int>(heads_each(a.B, a.H));
    a.by_together = fast_div(static_cast<uint32_t>(std::min<int64_t>(a.heads_each, kHeadsTogether)));
    a.by_blocks = fast_div(static_cast<uint32_t>(row_blocks(a.n_q)));
    a.by_heads = fast_div(a.H);
    const unsigned grid = static_cast<unsigned>(expanded_workgroups(a.B, a.n_q, a.H));
    if (a.d == 128) hipLaunchKernelGGL(k_expanded_attention<128>, dim3(grid), dim3(64 * kWavesExpanded), 0, s, a);
    else hipLaunchKernelGGL(k_expanded_attention<64>, dim3(grid), dim3(64 * kWavesExpanded), 0, s, a);
    return hipGetLastError();
}

}  // namespace cospec
