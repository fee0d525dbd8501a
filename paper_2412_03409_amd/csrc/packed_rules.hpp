// Which rows and keys of a paged or packed cache a call works on.  Plain integer rules, apart from the kernels so that they can be
// compiled and enumerated on the host.
#pragma once

#include <stdint.h>

namespace pkv {

// Rows of a sequence between its two offsets: none where these are not in 0 ... T.
__host__ __device__ __forceinline__ int new_rows(int first, int last, int T) { return first >= 0 && last <= T && last > first ? last - first : 0; }

// Keys that some of the first `rows` of a sequence's n new rows see, when its segment holds `len` (the new rows' own among them): row i
// sees the first len - n + i + 1.  A sequence without rows in the call sees none, however many its cache holds: nothing is read for it.
__host__ __device__ __forceinline__ int keys_seen(int rows, int n, int len) {
    const int end = len - n + rows;
    return rows <= 0 || end <= 0 ? 0 : end < len ? end : len;
}

}  // namespace pkv
