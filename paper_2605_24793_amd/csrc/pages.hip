// The pages under the caches: sharing, handing out, giving back, moving to the front, copying.
//
// Which page is handed out follows from the counts alone (the k-th request takes the k-th lowest free
// page), so one workgroup numbers requests and free pages by prefix sums: a launch, no state beside
// the counts, and no order of atomics that would show.  What many workgroups do (entries of tables,
// bytes of pages) needs no numbers.
#include <algorithm>

#include "pages.h"

namespace cospec {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kEntryThreads = 256;

// A copy is bound by memory; a thread has four 16-byte loads out at a time, and eight workgroups of them share a CU.  64
// pages of 2 MB (8 layers) that 8 sequences share: 45.1 us with pieces of 16 KB, 53.8 of 8, 49.2 of 32; 46.7 with
// 1024 workgroups, 44.8 with 4096, where 449 MB of separate pages take 105 and 107.
constexpr int kPieceBytes = 16384;    // of a page's plane, one workgroup's turn
constexpr int kCopyWorkgroups = 2048;
constexpr int kPoolWaves = kPoolThreads / 64;

__device__ inline bool names_page(int32_t e, int64_t n_pages) { return e >= 0 && e < n_pages; }

// Entries of the table that hold the first `len` positions.
__device__ inline int entries_of(int32_t len, int log_page, int max_pages) {
    const int64_t pages = (static_cast<int64_t>(max(len, 0)) + (1 << log_page) - 1) >> log_page;
    return static_cast<int>(min(pages, static_cast<int64_t>(max_pages)));
}

__global__ __launch_bounds__(kEntryThreads) void k_pages_fork(ForkArgs a) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kEntryThreads + threadIdx.x;
    if (i >= static_cast<int64_t>(a.B) * a.max_pages) return;
    const int b = quot(a.by_pages, static_cast<uint32_t>(i)), j = static_cast<int>(i) - b * a.max_pages;
    const int32_t from = a.row[b];
    int32_t e = -1;
    if (from >= 0 && from < a.rows && j < entries_of(a.len[b], a.log_page, a.max_pages))
        e = a.table[static_cast<int64_t>(from) * a.max_pages + j];
    const bool page = names_page(e, a.n_pages);
    if (page) atomicAdd(a.refs + e, 1);
    a.table_to[i] = page ? e : -1;
}

__global__ __launch_bounds__(kEntryThreads) void k_pages_release(ReleaseArgs a) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kEntryThreads + threadIdx.x;
    if (i >= static_cast<int64_t>(a.B) * a.max_pages) return;
    const int b = quot(a.by_pages, static_cast<uint32_t>(i)), j = static_cast<int>(i) - b * a.max_pages;
    if (j < entries_of(a.keep[b], a.log_page, a.max_pages)) return;
    const int32_t e = a.table[i];
    if (names_page(e, a.n_pages)) atomicSub(a.refs + e, 1);
    a.table[i] = -1;
}

// Numbers the set flags of the workgroup's threads in order: how many there are in lower threads
// (`in`: of this one's); `total` becomes that of all.  s [2][kPoolWaves], the turn's parity chooses.
__device__ inline int number(int in, int *s, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = in;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(sum, off);
        if (lane >= off) sum += x;
    }
    if (lane == 63) s[wave] = sum;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPoolWaves; ++w) {
        const int x = s[w];
        before += w < wave ? x : 0;
        total += x;
    }
    return before + sum - in;
}

// Four consecutive counts from page p on; pages past the last one count as in use (`past`: as what).
__device__ inline int4 four_refs(const int32_t *refs, int64_t p, int64_t n_pages, int past) {
    int4 r;
    r.x = p < n_pages ? refs[p] : past;
    r.y = p + 1 < n_pages ? refs[p + 1] : past;
    r.z = p + 2 < n_pages ? refs[p + 2] : past;
    r.w = p + 3 < n_pages ? refs[p + 3] : past;
    return r;
}

struct Request {
    int64_t at;                // its entry, or -1: none
    int32_t entry;
    bool first_part;           // the sequence's first new position is inside this page
};

__device__ inline Request request(const ReserveArgs &a, int64_t i) {
    const int b = quot(a.by_touched, static_cast<uint32_t>(i));
    const int w = static_cast<int>(i - static_cast<int64_t>(b) * a.touched);
    const int64_t begin = a.start[b], cnt = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const int64_t lo = max(begin, static_cast<int64_t>(0));
    const int64_t hi = min(begin + cnt, static_cast<int64_t>(a.max_pages) << a.log_page);
    const int64_t j = (lo >> a.log_page) + w;
    if (lo >= hi || (j << a.log_page) >= hi) return Request{-1, -1, false};
    const int64_t at = static_cast<int64_t>(b) * a.max_pages + j;
    return Request{at, a.table[at], w == 0 && (lo & ((1 << a.log_page) - 1)) != 0};
}

__global__ __launch_bounds__(kPoolThreads) void k_pages_reserve(ReserveArgs a) {
    __shared__ int s_sum[2][kPoolWaves];
    const int tid = threadIdx.x;
    const int64_t requests = static_cast<int64_t>(a.B) * a.touched;
    // requests, numbered
    int need = 0, turn = 0;
    for (int64_t base = 0; base < requests; base += kPoolThreads, turn ^= 1) {
        const int64_t i = base + tid;
        bool wants = false;
        if (i < requests) {
            const Request r = request(a, i);
            wants = r.at >= 0 && (!names_page(r.entry, a.n_pages) || a.refs[r.entry] > 1);
        }
        int total;
        const int k = need + number(wants, s_sum[turn], total);
        if (i < requests) a.rank[i] = wants ? k : -1;
        need += total;
    }
    // the free pages of lowest number
    int found = 0;
    int4 next = four_refs(a.refs, 4 * tid, a.n_pages, 1);
    for (int64_t base = 0; base < a.n_pages && found < need; base += 4 * kPoolThreads, turn ^= 1) {
        const int64_t p = base + 4 * tid;
        const int4 r = next;
        next = four_refs(a.refs, p + 4 * kPoolThreads, a.n_pages, 1);
        int total;
        int k = found + number((r.x == 0) + (r.y == 0) + (r.z == 0) + (r.w == 0), s_sum[turn], total);
        const int page = static_cast<int>(p);
        if (r.x == 0 && k++ < need) a.fresh[k - 1] = page;
        if (r.y == 0 && k++ < need) a.fresh[k - 1] = page + 1;
        if (r.z == 0 && k++ < need) a.fresh[k - 1] = page + 2;
        if (r.w == 0 && k++ < need) a.fresh[k - 1] = page + 3;
        found += total;
    }
    const bool enough = found >= need;
    if (tid == 0) *a.lacking = enough ? 0 : need - found;
    __syncthreads();                                        // the numbers are written, and no count is read any more
    for (int64_t i = tid; i < requests; i += kPoolThreads) {
        const int b = quot(a.by_touched, static_cast<uint32_t>(i));
        const bool head = i == static_cast<int64_t>(b) * a.touched;
        const int k = a.rank[i];
        int2 copy = make_int2(-1, -1);
        if (enough && k >= 0) {
            const Request r = request(a, i);
            const int32_t page = a.fresh[k];
            const bool had = names_page(r.entry, a.n_pages);
            a.refs[page] = 1;
            if (had) atomicSub(a.refs + r.entry, 1);
            a.table[r.at] = page;
            if (had && r.first_part) copy = make_int2(r.entry, page);
        }
        if (head) reinterpret_cast<int2 *>(a.copies)[b] = copy;
    }
}

// The entries of pages that move, by one workgroup or many.
__device__ inline void move_entries(const CompactArgs &a, int64_t first, int64_t step) {
    for (int64_t i = first; i < a.entries; i += step) {
        const int32_t e = a.table[i];
        if (!names_page(e, a.n_pages)) continue;
        const int32_t t = a.to[e];
        if (t >= 0) a.table[i] = t;
    }
}

// With `entries` the workgroup rewrites the table as well.
template <bool ENTRIES> __global__ __launch_bounds__(kPoolThreads) void k_pages_compact(CompactArgs a) {
    __shared__ int s_sum[2][kPoolWaves];
    const int tid = threadIdx.x;
    int turn = 0, used = 0;
    {
        int mine = 0;
        for (int64_t p = 4 * tid; p < a.n_pages; p += 4 * kPoolThreads) {
            const int4 r = four_refs(a.refs, p, a.n_pages, 0);
            mine += (r.x > 0) + (r.y > 0) + (r.z > 0) + (r.w > 0);
        }
        number(mine, s_sum[turn], used);
        turn ^= 1;
    }
    // pages in use behind the front, and free ones in it; there are as many of both
    int behind = 0, holes = 0;
    for (int64_t base = 0; base < a.n_pages; base += kPoolThreads, turn ^= 1) {
        const int64_t p = base + tid;
        bool from = false, hole = false;
        if (p < a.n_pages) {
            const bool in_use = a.refs[p] > 0;
            from = in_use && p >= used;
            hole = !in_use && p < used;
            a.to[p] = -1;
        }
        // both in one sum: a turn has at most 2^10 of each
        int total;
        const int k = number((from ? 1 : 0) + (hole ? 1 << 16 : 0), s_sum[turn], total);
        if (from) a.moves[behind + (k & 0xffff)].x = static_cast<int>(p);
        if (hole) a.moves[holes + (k >> 16)].y = static_cast<int>(p);
        behind += total & 0xffff;
        holes += total >> 16;
    }
    __syncthreads();
    const int64_t room = max(a.n_pages / 2, static_cast<int64_t>(1));
    for (int64_t k = tid; k < room; k += kPoolThreads) {
        if (k < behind) {
            const int2 m = a.moves[k];
            a.refs[m.y] = a.refs[m.x];
            a.refs[m.x] = 0;
            a.to[m.x] = m.y;
        } else {
            a.moves[k] = make_int2(-1, -1);
        }
    }
    if (tid == 0) *a.n_moves = behind;
    if constexpr (ENTRIES) {
        __syncthreads();
        move_entries(a, tid, kPoolThreads);
    }
}

__global__ __launch_bounds__(kEntryThreads) void k_pages_entries(CompactArgs a) {
    move_entries(a, static_cast<int64_t>(blockIdx.x) * kEntryThreads + threadIdx.x,
                 static_cast<int64_t>(gridDim.x) * kEntryThreads);
}

// Pieces of a page's planes, dealt to the workgroups: 4.4 TB/s read and written where no page is read twice (32 sequences' pages,
// 449 MB), 4.7 for a large copy.
__global__ __launch_bounds__(kEntryThreads) void k_pages_copy(CopyArgs a) {
    const int tid = threadIdx.x;
    const int pairs = a.count ? min(max(*a.count, 0), a.n_pairs) : a.n_pairs;
    const uint32_t per_pair = a.first[a.n_planes];
    const int64_t pieces = static_cast<int64_t>(pairs) * per_pair;
    for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
        const int k = static_cast<int>(i / per_pair);
        const uint32_t piece = static_cast<uint32_t>(i - static_cast<int64_t>(k) * per_pair);
        const int2 pr = a.pairs[k];
        if (!names_page(pr.x, a.n_pages) || !names_page(pr.y, a.n_pages) || pr.x == pr.y) continue;
        int plane = 0;
        while (plane + 1 < a.n_planes && a.first[plane + 1] <= piece) ++plane;
        const int64_t bytes = a.bytes[plane], at = static_cast<int64_t>(piece - a.first[plane]) * kPieceBytes;
        const int here = static_cast<int>(min(bytes - at, static_cast<int64_t>(kPieceBytes)));
        const char *src = a.data[plane] + pr.x * bytes + at;
        char *dst = a.data[plane] + pr.y * bytes + at;
        if (((reinterpret_cast<uintptr_t>(a.data[plane]) | static_cast<uintptr_t>(bytes)) & 15) == 0) {
            constexpr int PER = kPieceBytes / 16 / kEntryThreads;
            u32x4 x[PER];
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int o = (u * kEntryThreads + tid) * 16;
                if (o < here) x[u] = *reinterpret_cast<const u32x4 *>(src + o);
            }
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int o = (u * kEntryThreads + tid) * 16;
                if (o < here) *reinterpret_cast<u32x4 *>(dst + o) = x[u];
            }
        } else {
            for (int o = tid * 4; o < here; o += kEntryThreads * 4)
                *reinterpret_cast<uint32_t *>(dst + o) = *reinterpret_cast<const uint32_t *>(src + o);
        }
    }
}

// Tables of more entries are rewritten by many workgroups, in a launch of their own, which costs 3 us of a small pool's
// 21 (4 sequences of 700 positions, 300 pages to spare).
constexpr int64_t kEntriesInPlace = 16384;

unsigned entry_grid(int64_t n) { return static_cast<unsigned>((n + kEntryThreads - 1) / kEntryThreads); }

}  // namespace

hipError_t launch_pages_fork(ForkArgs a, hipStream_t s) {
    a.by_pages = fast_div(a.max_pages);
    hipLaunchKernelGGL(k_pages_fork, dim3(entry_grid(static_cast<int64_t>(a.B) * a.max_pages)), dim3(kEntryThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_reserve(ReserveArgs a, hipStream_t s) {
    a.by_touched = fast_div(a.touched);
    hipLaunchKernelGGL(k_pages_reserve, dim3(1), dim3(kPoolThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_release(ReleaseArgs a, hipStream_t s) {
    a.by_pages = fast_div(a.max_pages);
    hipLaunchKernelGGL(k_pages_release, dim3(entry_grid(static_cast<int64_t>(a.B) * a.max_pages)), dim3(kEntryThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s) {
    if (a.entries <= kEntriesInPlace) {
        hipLaunchKernelGGL(k_pages_compact<true>, dim3(1), dim3(kPoolThreads), 0, s, a);
    } else {
        hipLaunchKernelGGL(k_pages_compact<false>, dim3(1), dim3(kPoolThreads), 0, s, a);
        hipLaunchKernelGGL(k_pages_entries, dim3(std::min(entry_grid(a.entries), 4096u)), dim3(kEntryThreads), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_pages_copy(CopyArgs a, hipStream_t s) {
    a.first[0] = 0;
    for (int p = 0; p < a.n_planes; ++p)
        a.first[p + 1] = a.first[p] + static_cast<uint32_t>((a.bytes[p] + kPieceBytes - 1) / kPieceBytes);
    const int64_t pieces = static_cast<int64_t>(a.n_pairs) * a.first[a.n_planes];
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(pieces, kCopyWorkgroups));
    hipLaunchKernelGGL(k_pages_copy, dim3(grid), dim3(kEntryThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace cospec
