// Page tables and slots of a paged cache from lengths.  A segment is one (sequence, layer): every layer keeps another number
// of positions, so every layer has its own row of the table.
//
//   held = ceil(old / ps), want = ceil(new / ps);  pages taken = max(0, want - held), given back = max(0, held - want);
//   first[i] = pages that the segments before i take (or give back): an exclusive sum over the segments in (s,l) order;
//   taken:       table[i, held + j] = ring[(head + first + j) mod P]
//   given back:  ring[(head + count + first + j) mod P] = table[i, want + j]
//   slot of a new row = page * ps + row in the page
//
// Free pages wait in a ring and not on a stack: what a call takes (at the head) and what it gives back (behind the end) are
// disjoint places, so that all entries move at once, in any order, with the same result.  (Ends of the ring without room for what
// comes back, which no sequence of calls leads to, are refused.)
// Bound: latency.  The sums need every length before the first entry can move; one workgroup of 1024 threads forms them (a
// sum of two counts by wavefront shuffles, the wavefronts' totals through LDS).  While what has to move is little the same
// workgroup moves it (SMALL: one launch), else a second launch spreads it over the chip.  64 sequences of 32 layers, a row each:
// 7.2 us, of which 3 go to the scattered table entries that one compute unit reads (all of them asked for next to the sums: 8.7).
// 64 sequences of 40 layers resized: 4.2 + 4.2.
#include "packed.hpp"
#include "fast_div.hpp"
#include "packed_rules.hpp"

namespace pkv {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kSmallSegs = 4096;        // segments whose records fit the planning workgroup's LDS
constexpr int kSmallSlots = 16384;      // slots, or places of the table, that the planning workgroup looks after itself
constexpr int kSlotThreads = 256;

struct PageParams {
    int S, T, layers, n;                // n = S * layers segments
    int num_pages, max_pages, shift;    // shift: log2 of the page size
    FastDiv by_layers, by_t, by_width;
    const int32_t *target, *row_off, *lens;
    int32_t *table, *ring;
    const int32_t* state;
    int32_t *lens_out, *state_out;
    int64_t* slots;
    int32_t* status;
    int4* head;                         // workspace: {accepted, head, count, 0}
    int2* rec;                          // workspace: {old length, first} of every segment
};

__device__ __forceinline__ int pages_of(const PageParams& p, int len) { return (len + (1 << p.shift) - 1) >> p.shift; }
__device__ __forceinline__ int ring_at(const PageParams& p, uint32_t at) { return ring_place(at, p.num_pages); }

// the sequence of row t: the last one that begins at t or before it (sequences without rows are passed over)
__device__ __forceinline__ int sequence_of(const int* off, int S, int t) {
    int lo = 0, hi = S;                 // off[lo] <= t < off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// Slot of row t in layer l.  The first entry of a page that was taken for it also enters the page into the table: every such
// page begins with a new row.
__device__ __forceinline__ int64_t give_slot(const PageParams& p, const int4& hd, const int2& r, int seg, int at) {
    const int held = pages_of(p, r.x), pos = r.x + at, page = pos >> p.shift, row = pos & ((1 << p.shift) - 1);
    int32_t* entry = p.table + (int64_t)seg * p.max_pages + page;
    int id;
    if (page < held) id = *entry;
    else {
        id = p.ring[ring_at(p, (uint32_t)hd.y + (uint32_t)r.y + (uint32_t)(page - held))];
        if (row == 0) *entry = id;
    }
    return ((int64_t)id << p.shift) + row;
}

constexpr int kPer = 4;                 // segments of a thread: 4096 in a round

template <bool APPEND, bool SMALL>
__global__ void __launch_bounds__(kPlanThreads)
page_plan_kernel(PageParams p) {
    __shared__ int2 s_sum[2][kPlanWaves];
    __shared__ int s_bad;
    __shared__ int2 s_rec[SMALL ? kSmallSegs : 1];
    __shared__ int s_off[APPEND && SMALL ? kMaxS + 1 : 1];
    __shared__ int s_len[!APPEND && SMALL ? kSmallSegs : 1];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const int limit = p.max_pages << p.shift;
    if (tid == 0) s_bad = 0;
    if constexpr (APPEND && SMALL)
        for (int i = tid; i <= p.S; i += kPlanThreads) s_off[i] = p.row_off[i];
    const int head = p.state[0], count = p.state[1];
    int2 carry = make_int2(0, 0);
    bool bad = false;
    int len[kPer];                      // new lengths (SMALL: there is one round)
    // Two rounds' sums alternate in LDS, so that one barrier per round is enough.
    for (int base = 0, turn = 0; base < p.n; base += kPlanThreads * kPer, turn ^= 1) {
        const int i0 = base + tid * kPer;
        int old[kPer];
        int2 mine[kPer], sum = make_int2(0, 0);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = i0 + e;
            old[e] = len[e] = 0;
            bool wrong = false;
            if (i < p.n) {
                old[e] = p.lens[i];
                if constexpr (APPEND) {
                    const int s = div_mod(i, p.by_layers).q;
                    const int a = p.row_off[s], b = p.row_off[s + 1];
                    wrong = a < 0 || b < a || b > p.T;
                    len[e] = wrong ? old[e] : old[e] + (b - a);    // lengths stay below 2^20 + 2^22
                } else {
                    len[e] = p.target[i];
                }
                wrong = wrong || old[e] < 0 || old[e] > limit || len[e] < 0 || len[e] > limit;
            }
            bad = bad || wrong;
            const int diff = wrong ? 0 : pages_of(p, len[e]) - pages_of(p, old[e]);
            mine[e] = make_int2(max(diff, 0), max(-diff, 0));
            sum.x += mine[e].x; sum.y += mine[e].y;
        }
        int2 incl = sum;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int ux = __shfl_up(incl.x, d, kWave), uy = __shfl_up(incl.y, d, kWave);
            if (lane >= d) { incl.x += ux; incl.y += uy; }
        }
        if (lane == kWave - 1) s_sum[turn][wv] = incl;
        if (turn == 0 && base == 0) __syncthreads();               // s_bad is cleared
        if (bad) s_bad = 1;
        __syncthreads();
        int2 before = make_int2(carry.x + incl.x - sum.x, carry.y + incl.y - sum.y);
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
            const int2 x = s_sum[turn][w];
            if (w < wv) { before.x += x.x; before.y += x.y; }
            carry.x += x.x; carry.y += x.y;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            if (i0 + e < p.n) {
                const int2 r = make_int2(old[e], mine[e].x > 0 ? before.x : before.y);
                if constexpr (SMALL) s_rec[i0 + e] = r; else p.rec[i0 + e] = r;
                if constexpr (SMALL && !APPEND) s_len[i0 + e] = len[e];
            }
            before.x += mine[e].x; before.y += mine[e].y;
        }
    }
    __syncthreads();
    const bool range = s_bad != 0 || ring_range(head, count, carry.y, p.num_pages);
    const bool few = carry.x > count;
    const bool ok = !range && !few;
    const int4 hd = make_int4(ok ? 1 : 0, head, count, 0);
    // (every thread has read what it needs of lens and state in front of the barrier: lens_out and state_out may be the same)
    if constexpr (SMALL) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int i = tid * kPer + e;
            if (i < p.n) p.lens_out[i] = ok ? len[e] : s_rec[i].x;
        }
    } else {
        for (int i = tid; i < p.n; i += kPlanThreads) {
            int n = p.rec[i].x;
            if (ok) {
                if constexpr (APPEND) {
                    const int s = div_mod(i, p.by_layers).q;
                    n += p.row_off[s + 1] - p.row_off[s];
                } else {
                    n = p.target[i];
                }
            }
            p.lens_out[i] = n;
        }
    }
    if (tid == 0) {
        p.state_out[0] = ok ? ring_at(p, (uint32_t)head + (uint32_t)carry.x) : head;
        p.state_out[1] = ok ? count - carry.x + carry.y : count;
        *p.status = range ? PKV_PAGES_RANGE : few ? PKV_PAGES_SHORT : 0;
        if constexpr (!SMALL) *p.head = hd;
    }
    if constexpr (!APPEND && SMALL) {
        if (!ok) return;
        // a thread per place of the table
        for (int x = tid; x < p.n * p.max_pages; x += kPlanThreads) {
            const DivMod sj = div_mod(x, p.by_width);
            const int2 r = s_rec[sj.q];
            const int held = pages_of(p, r.x), want = pages_of(p, s_len[sj.q]), j = sj.r;
            if (j >= held && j < want) p.table[x] = p.ring[ring_at(p, (uint32_t)hd.y + (uint32_t)r.y + (uint32_t)(j - held))];
            if (j >= want && j < held)
                p.ring[ring_at(p, (uint32_t)hd.y + (uint32_t)hd.z + (uint32_t)r.y + (uint32_t)(j - want))] = p.table[x];
        }
    }
    if constexpr (APPEND && SMALL) {
        const int total = p.layers * p.T;
#pragma unroll 2
        for (int x = tid; x < total; x += kPlanThreads) {
            const DivMod lt = div_mod(x, p.by_t);      // layer, row
            int64_t slot = -1;
            if (ok && lt.r >= s_off[0] && lt.r < s_off[p.S]) {
                const int s = sequence_of(s_off, p.S, lt.r), seg = s * p.layers + lt.q;
                slot = give_slot(p, hd, s_rec[seg], seg, lt.r - s_off[s]);
            }
            p.slots[x] = slot;
        }
    }
}

// slots of 256 rows in a few layers
__global__ void __launch_bounds__(kSlotThreads)
page_slots_kernel(PageParams p, int per) {
    __shared__ int s_off[kMaxS + 1];
    for (int i = threadIdx.x; i <= p.S; i += kSlotThreads) s_off[i] = p.row_off[i];
    __syncthreads();
    const int t = blockIdx.x * kSlotThreads + threadIdx.x;
    if (t >= p.T) return;
    const int4 hd = *p.head;
    const bool real = hd.x != 0 && t >= s_off[0] && t < s_off[p.S];
    const int s = real ? sequence_of(s_off, p.S, t) : 0, at = t - s_off[s];
    const int l0 = blockIdx.y * per, l1 = min(p.layers, l0 + per);
#pragma unroll 4
    for (int l = l0; l < l1; ++l) {
        const int seg = s * p.layers + l;
        p.slots[(int64_t)l * p.T + t] = real ? give_slot(p, hd, p.rec[seg], seg, at) : -1;
    }
}

// a wavefront moves the pages of a segment
__global__ void __launch_bounds__(kSlotThreads)
page_move_kernel(PageParams p) {
    const int seg = blockIdx.x * (kSlotThreads / kWave) + threadIdx.x / kWave;
    if (seg >= p.n) return;
    const int4 hd = *p.head;
    if (hd.x == 0) return;
    const int2 r = p.rec[seg];
    const int held = pages_of(p, r.x), want = pages_of(p, p.target[seg]), lane = threadIdx.x & (kWave - 1);
    int32_t* row = p.table + (int64_t)seg * p.max_pages;
#pragma unroll 4
    for (int j = held + lane; j < want; j += kWave) row[j] = p.ring[ring_at(p, (uint32_t)hd.y + (uint32_t)r.y + (uint32_t)(j - held))];
#pragma unroll 4
    for (int j = want + lane; j < held; j += kWave)
        p.ring[ring_at(p, (uint32_t)hd.y + (uint32_t)hd.z + (uint32_t)r.y + (uint32_t)(j - want))] = row[j];
}

size_t page_ws_bytes(int S, int layers) { return 256 + (size_t)S * layers * sizeof(int2); }

hipError_t launch_pages(int S, int T, const pkv_paging& g, const int32_t* target, const int32_t* row_off, const int32_t* lens,
                        int32_t* table, int32_t* ring, const int32_t* state, int32_t* lens_out, int32_t* state_out,
                        int64_t* slots, int32_t* status, void* ws, hipStream_t st) {
    PageParams p;
    p.S = S; p.T = T; p.layers = g.layers; p.n = S * g.layers;
    p.num_pages = g.num_pages; p.max_pages = g.max_pages; p.shift = __builtin_ctz((unsigned)g.page_size);
    p.by_layers = fast_div(g.layers); p.by_t = fast_div(T > 0 ? T : 1); p.by_width = fast_div(g.max_pages);
    p.target = target; p.row_off = row_off; p.lens = lens; p.table = table; p.ring = ring; p.state = state;
    p.lens_out = lens_out; p.state_out = state_out; p.slots = slots; p.status = status;
    p.head = (int4*)ws; p.rec = (int2*)((char*)ws + 256);
    const bool segs = p.n <= kSmallSegs;
    if (row_off) {
        if (segs && (int64_t)g.layers * T <= kSmallSlots) {
            hipLaunchKernelGGL((page_plan_kernel<true, true>), dim3(1), dim3(kPlanThreads), 0, st, p);
        } else {
            hipLaunchKernelGGL((page_plan_kernel<true, false>), dim3(1), dim3(kPlanThreads), 0, st, p);
            const int per = 8;
            hipLaunchKernelGGL(page_slots_kernel, dim3((T + kSlotThreads - 1) / kSlotThreads, (g.layers + per - 1) / per),
                               dim3(kSlotThreads), 0, st, p, per);
        }
    } else if (segs && (int64_t)p.n * g.max_pages <= kSmallSlots) {
        hipLaunchKernelGGL((page_plan_kernel<false, true>), dim3(1), dim3(kPlanThreads), 0, st, p);
    } else {
        hipLaunchKernelGGL((page_plan_kernel<false, false>), dim3(1), dim3(kPlanThreads), 0, st, p);
        hipLaunchKernelGGL(page_move_kernel, dim3((p.n + kSlotThreads / kWave - 1) / (kSlotThreads / kWave)), dim3(kSlotThreads),
                           0, st, p);
    }
    return hipGetLastError();
}

}  // namespace pkv
