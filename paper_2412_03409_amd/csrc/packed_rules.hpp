// Which rows and keys of a paged or packed cache a call works on, what the ring of free pages can give and take, and how many
// workgroups a compaction has.  Plain integer rules, apart from the kernels so that they can be compiled and enumerated on the host.
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

// Ends of the ring that cannot be, for a call that gives `given` pages back: the places behind the end that it puts them into must be
// free before the call, so that they are disjoint from those it takes from at the head, and none lies a second turn ahead.  (Pages that
// segments hold are not in the ring, so ends that are possible always have that room.)
__host__ __device__ __forceinline__ bool ring_range(int head, int count, int given, int num_pages) {
    return head < 0 || head >= num_pages || count < 0 || count > num_pages || (int64_t)count + given > num_pages;
}
// The place `at` places behind place 0, for at < 2 num_pages: head + i for i < taken, head + count + i for i < given.
__host__ __device__ __forceinline__ int ring_place(uint32_t at, int num_pages) {
    return (int)(at >= (uint32_t)num_pages ? at - (uint32_t)num_pages : at);
}

// Workgroups per (segment, kv head): one per 64-row chunk up to 16 chunks (1024 rows), made odd.  The hardware
// deals consecutive workgroups out to the eight XCDs in turn; with an even count -- 16 above all -- chunk c of
// every (segment, head) lands on the same XCD, and since most segments keep few rows the XCDs of the high
// chunk indices see hardly any work (measured with 16: 2.3 instead of 4.3 TB/s from N = 1000 on).
inline int gather_chunks(int N) {
    const int all_chunks = (N + 63) / 64;
    const int nchunk = all_chunks < 16 ? all_chunks : 16;
    return nchunk | 1;
}

// Workgroups of a launch: below 2^24, as a grid's threads (256 of a workgroup) are counted in 32 bits.
inline long long gather_workgroups(int N, int Hkv, long long segments) { return gather_chunks(N) * (long long)Hkv * segments; }
inline bool gather_fits(int N, int Hkv, long long segments) { return gather_workgroups(N, Hkv, segments) < 1ll << 24; }

}  // namespace pkv
