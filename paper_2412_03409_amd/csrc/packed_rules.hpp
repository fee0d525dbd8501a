// Which rows and keys of a paged or packed cache a call works on, and what the ring of free pages can give and take.  Plain integer
// rules, apart from the kernels so that they can be compiled and enumerated on the host.
#pragma once

#include <stdint.h>

#include "../../include/prefixkv.h"

namespace pkv {

// Rows of a sequence between its two offsets: none where these are not in 0 ... T.
__host__ __device__ __forceinline__ int new_rows(int first, int last, int T) { return first >= 0 && last <= T && last > first ? last - first : 0; }

// Keys that some of the first `rows` of a sequence's n new rows see, when its segment holds `len` (the new rows' own among them): row i
// sees the first len - n + i + 1.  A sequence without rows in the call sees none, however many its cache holds: nothing is read for it.
__host__ __device__ __forceinline__ int keys_seen(int rows, int n, int len) {
    const int end = len - n + rows;
    return rows <= 0 || end <= 0 ? 0 : end < len ? end : len;
}

// Whether a call may take `taken` pages from the head of the ring and put `given` behind its end: 0, or why not.  The places it puts
// them into must be free before the call, too: they are disjoint from those it takes from, and none lies a second turn ahead.  (Pages
// that segments hold are not in the ring, so ends that are possible always have that room.)
__host__ __device__ __forceinline__ int ring_verdict(int head, int count, int taken, int given, int num_pages) {
    if (head < 0 || head >= num_pages || count < 0 || count > num_pages || given > num_pages - count) return PKV_PAGES_RANGE;
    return taken > count ? PKV_PAGES_SHORT : 0;
}
// The place `at` places behind place 0, for at < 2 num_pages: head + i for i < taken, head + count + i for i < given.
__host__ __device__ __forceinline__ int ring_place(uint32_t at, int num_pages) {
    return (int)(at >= (uint32_t)num_pages ? at - (uint32_t)num_pages : at);
}

}  // namespace pkv
