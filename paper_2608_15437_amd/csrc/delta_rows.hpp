// Rows of a chunk of the gated delta rule, in 32 bits: an array may have 2^31 - 1 of them, so what is added to a row is
// compared with what is left behind it first.
#pragma once

#include <stdint.h>

namespace mmbev {

constexpr int kDeltaRows = 32;  // rows of a chunk

// Chunks of [lo, hi), lo <= hi.
constexpr int32_t delta_chunks(int32_t lo, int32_t hi) { return (hi - lo) / kDeltaRows + ((hi - lo) % kDeltaRows != 0); }

// First row of chunk c.
constexpr int32_t delta_chunk(int32_t lo, int32_t c) { return lo + c * kDeltaRows; }

// Whether the i-th row from s0 on lies before hi, and that row or the last one before hi; s0 < hi.
constexpr bool delta_row_there(int32_t s0, int32_t i, int32_t hi) { return i < hi - s0; }
constexpr int32_t delta_row(int32_t s0, int32_t i, int32_t hi) { return s0 + (i < hi - s0 - 1 ? i : hi - s0 - 1); }

}  // namespace mmbev
