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

}  // namespace cospec
