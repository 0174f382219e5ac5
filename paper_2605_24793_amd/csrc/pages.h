// The pages under the caches: arguments of the kernels of pages.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace cospec {

constexpr int kPoolThreads = 1024;    // the one workgroup that numbers pages
constexpr int kMaxPlanes = 64;        // of a launch: what the kernel's arguments hold

struct ForkArgs {
    int32_t *refs;
    int64_t n_pages;
    const int32_t *table, *row, *len;
    int32_t rows, B, max_pages, log_page;
    int32_t *table_to;
    FastDiv by_pages;          // set by the launch
};

struct ReserveArgs {
    int32_t *refs;
    int64_t n_pages;
    int32_t *table;
    const int32_t *start, *count;
    int32_t B, n, max_pages, log_page;
    int32_t touched;           // pages that n positions can touch
    int32_t *copies, *lacking;
    int32_t *rank, *fresh;     // workspace: [B * touched] each
    FastDiv by_touched;        // set by the launch
};

struct ReleaseArgs {
    int32_t *refs;
    int64_t n_pages;
    int32_t *table;
    const int32_t *keep;
    int32_t B, max_pages, log_page;
    FastDiv by_pages;          // set by the launch
};

struct CompactArgs {
    int32_t *refs;
    int64_t n_pages;
    int32_t *table;
    int64_t entries;           // of the table
    int2 *moves;
    int32_t *n_moves;
    int32_t *to;               // workspace [n_pages]: where a page goes, or -1
};

struct CopyArgs {
    int64_t n_pages;
    const int2 *pairs;
    int32_t n_pairs;
    const int32_t *count;      // or null
    int32_t n_planes;
    char *data[kMaxPlanes];
    int64_t bytes[kMaxPlanes];
    uint32_t first[kMaxPlanes + 1];   // first piece of a plane's page among those of a pair
};

hipError_t launch_pages_fork(ForkArgs a, hipStream_t s);
hipError_t launch_pages_reserve(ReserveArgs a, hipStream_t s);
hipError_t launch_pages_release(ReleaseArgs a, hipStream_t s);
hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s);
hipError_t launch_pages_copy(CopyArgs a, hipStream_t s);   // `first` is set here

}  // namespace cospec
