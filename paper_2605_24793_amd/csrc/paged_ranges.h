// Ranges of the paged cache's kernels that follow from lengths in device memory, where any 32-bit value may
// stand.  constexpr: of the host and the device alike.
#pragma once

#include <stdint.h>

namespace cospec {

// What an append of tokens 0 .. count - 1 to positions start .. does to page j of a sequence: places [lo, hi) are
// new (none if lo >= hi), and place s takes token base + s.
struct NewPlaces {
    int64_t base;
    int lo, hi;
};

constexpr NewPlaces new_places(int64_t start, int64_t count, int64_t j, int log_page) {
    const int64_t P = static_cast<int64_t>(1) << log_page, base = j * P - start;
    const int64_t lo = base < 0 ? -base : 0, hi = count - base;
    // clamped in 64 bits: a start far below position 0 puts hi past what 32 hold
    return NewPlaces{base, static_cast<int>(lo < P ? lo : P), static_cast<int>(hi < 0 ? 0 : hi < P ? hi : P)};
}

// Keys [0, kend) cut into `count` pieces (at least one) of `chunk` keys, the last one shorter; `part`: the keys of
// an even share, `step`: what a chunk is a multiple of, `least`: its least length.
struct Pieces {
    int chunk, count;
};

constexpr Pieces pieces_of(int kend, int part, int step, int least) {
    const int even = (part + step - 1) / step * step, chunk = even > least ? even : least;
    // (kend + chunk may be more than 31 bits hold)
    return Pieces{chunk, kend > 0 ? (kend - 1) / chunk + 1 : 1};
}

}  // namespace cospec
