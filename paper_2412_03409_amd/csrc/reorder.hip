// Places of a paged cache become what their beams continue.  Places come in groups of W, a group holds the beams of a prompt:
//   place (g,i) becomes what place (g, parents[g,i]) was, in every layer; -1: empty.
// Pages are shared, not copied: a page that is full is never written again.  The page that a length ends in is, so only the lowest
// place of those that continue one keeps it, and each other gets a page of its own with the used rows copied.  A page that no place
// holds any more goes back to the ring.
//
// Who shares a page can be read from the table itself: places share only what they had in common, at the same entry of the same layer.
// So a column, entry j of a layer in the W places of a group, says all about its pages:
//   kept(i)   some place's new entry is old(i)                       first(i)  no lower place has old(i) too
//   given back: old(i) that is not kept, by the first place that had it.
// W lanes have a column, and look at each other's entries by shuffles.
//
// What is given back goes to the ring in (place, layer, entry) order, what is taken comes from it in (place, layer) order: the sums of
// both over all segments lie between two launches.
//  reorder_count_kernel   counts both, a workgroup for a layer of a group, and notes what has to be copied from where.
//  reorder_sums_kernel    their sums, one workgroup; where there are few segments every workgroup of the next launch forms its own.
//  reorder_apply_kernel   the first workgroups rewrite the table and the ring, the others copy rows.
// Bound: latency for a request's beams, HBM where many partly filled pages are copied.  8 groups of 4 places, 32 layers of 8 heads of 128 in
// bf16, 80 MB read and written: 4.0 + 16.3 us (4.9 TB/s in the second); one group of 4: 4.0 + 6.4.
#include "packed.hpp"
#include "fast_div.hpp"
#include "packed_rules.hpp"

namespace pkv {

constexpr int kReorderThreads = 256;
constexpr int kReorderWaves = kReorderThreads / kWave;
constexpr int kSumThreads = 1024;
// Segments up to which a workgroup sums them up itself.  us, so / with a launch of its own, 4 places a group: 8 heads of 128, 512 segments 14.9 / 17.3,
// 1024 18.5 / 21.7, 1280 19.9 / 22.0, 1536 26.4 / 28.5, 2048 37.8 / 37.6, 4096 65.4 / 56.5; a head of 64, 128 segments 10.9 / 14.2, 1024 11.3 / 14.0, 1536 12.7 / 13.9,
// 2048 13.8 / 15.2, 4096 19.7 / 17.5 (groups of 8: 24.2 / 17.5).  They meet at about 2048: up to there this is 1 to 2 us too careful.
constexpr int kOwnSums = 1024;
constexpr int kCopyBytes = 32768;       // of a tensor that a workgroup copies

struct ReorderParams {
    int W, layers, n;                   // n = S * layers segments
    int lanes;                          // of a column: W, rounded up to a power of two
    int num_pages, max_pages, shift;
    int units, splits;                  // units: groups * layers; splits: workgroups that copy a segment's rows
    int Hkv, heads_per;                 // heads that a workgroup copies
    int row_bytes, row_shift;           // of an entry of one head; log2 of its 16-byte pieces
    FastDiv by_layers, by_splits;
    const int32_t *parents, *table, *lens;
    int32_t* ring;
    const int32_t* state;
    int32_t *table_out, *lens_out, *state_out;
    unsigned char *kp, *vp;
    int32_t* status;
    // workspace, in whole fours of segments
    int4* head;                         // {head, count, taken, given} (the latter two of all segments), {status, 0, 0, 0}
    int4* quarters;                     // pages that the wavefronts' columns of a segment give back
    int4* given;                        // their sums, four segments
    uint32_t* flags;                    // of four segments, a byte each: kTakes, kWrong
    int2* from;                         // where kTakes: the page to copy from, rows
    int2* first;                        // pages taken and given back by the segments before (reorder_sums_kernel)
};
constexpr uint32_t kTakes = 1, kWrong = 2;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// What a lane knows of its place: in every column the same.
struct GroupPlace {
    int w, col, s, parent;              // parent: lane of its column, -1
    bool real, again;                   // again: a lower place continues the same one
    int old_len, new_len;
};

__device__ __forceinline__ int pages_in(const ReorderParams& p, int len) { return (len + (1 << p.shift) - 1) >> p.shift; }

// -> false where a parent or a length cannot be (of the whole group's)
__device__ __forceinline__ bool look(const ReorderParams& p, int g, int l, int lane, GroupPlace& x) {
    x.w = lane & (p.lanes - 1);
    x.col = lane / p.lanes;
    x.real = x.w < p.W;
    x.s = g * p.W + min(x.w, p.W - 1);
    const int from = x.real ? p.parents[x.s] : -1;
    x.old_len = x.real ? p.lens[(int64_t)x.s * p.layers + l] : 0;
    const bool bad = from < -1 || from >= p.W || x.old_len < 0 || x.old_len > (p.max_pages << p.shift);
    if (__builtin_amdgcn_ballot_w64(bad) != 0) return false;
    x.parent = from;
    const int base = lane - x.w, len = __shfl(x.old_len, base + max(from, 0), kWave);
    x.new_len = from < 0 ? 0 : len;
    x.again = false;
    for (int c = 0; c < p.W; ++c) {
        const int other = __shfl(from, base + c, kWave);
        x.again = x.again || (c < x.w && other == from && from >= 0);
    }
    return true;
}
__device__ __forceinline__ bool copies(const ReorderParams& p, const GroupPlace& x) { return x.again && (x.new_len & ((1 << p.shift) - 1)) != 0; }

struct Column { int id, next; bool in_old, in_new, given; };     // old and new entry (next: of a copied page the one copied from)
__device__ __forceinline__ Column column(const ReorderParams& p, const GroupPlace& x, int l, int lane, int j) {
    Column c;
    c.in_old = j < pages_in(p, x.old_len);
    c.in_new = j < pages_in(p, x.new_len);
    c.id = c.in_old ? p.table[((int64_t)x.s * p.layers + l) * p.max_pages + j] : -1;
    const int base = lane - x.w, from = __shfl(c.id, base + max(x.parent, 0), kWave);
    c.next = from;
    const int holds = c.in_new && !(copies(p, x) && j == x.new_len >> p.shift) ? from : -2;
    bool kept = false, lower = false;
    for (int i = 0; i < p.W; ++i) {
        const int h = __shfl(holds, base + i, kWave), o = __shfl(c.id, base + i, kWave);
        kept = kept || h == c.id;
        lower = lower || (i < x.w && o == c.id);
    }
    c.given = c.in_old && (uint32_t)c.id < (uint32_t)p.num_pages && !kept && !lower;
    return c;
}
// the columns of a wavefront: a quarter, in steps of 64 / lanes
struct Range { int begin, end, step; };
__device__ __forceinline__ Range columns_of(const ReorderParams& p, const GroupPlace& x, int wv) {
    int most = max(pages_in(p, x.old_len), pages_in(p, x.new_len));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = max(most, __shfl_xor(most, d, kWave));
    const int step = kWave / p.lanes, each = (most + kReorderWaves * step - 1) / (kReorderWaves * step) * step;
    return {min(most, wv * each), min(most, (wv + 1) * each), step};
}
// pages that this wavefront's columns give back, of each place (in the lanes of column 0)
__device__ __forceinline__ int count_given(const ReorderParams& p, const GroupPlace& x, int l, int lane, const Range& r) {
    int given = 0;
    for (int j = r.begin; j < r.end; j += r.step) {
        const Column c = column(p, x, l, lane, j + x.col);
        given += c.given && j + x.col < r.end;
    }
    for (int d = p.lanes; d < kWave; d <<= 1) given += __shfl_xor(given, d, kWave);
    return given;
}

__global__ void __launch_bounds__(kReorderThreads)
reorder_count_kernel(ReorderParams p) {
    __shared__ __attribute__((aligned(16))) int s_given[kMaxBeams][kReorderWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const DivMod gl = uniform_div_mod((int)blockIdx.x, p.by_layers);
    const int g = gl.q, l = gl.r;
    if (blockIdx.x == 0) {
        if (tid == 0) p.head[0] = make_int4(p.state[0], p.state[1], 0, 0);
        if (tid >= p.n % 4 && tid < 4 && p.n % 4 != 0) {            // the last four's places behind the end
            ((uint8_t*)p.flags)[p.n - p.n % 4 + tid] = 0;
            ((int*)p.given)[p.n - p.n % 4 + tid] = 0;
        }
    }
    GroupPlace x;
    const bool ok = look(p, g, l, lane, x);
    if (ok) {
        const int given = count_given(p, x, l, lane, columns_of(p, x, wv));
        if (x.real && x.col == 0) s_given[x.w][wv] = given;
    }
    __syncthreads();
    if (wv != 0 || !x.real || x.col != 0) return;
    const int64_t seg = (int64_t)x.s * p.layers + l;
    uint32_t flags = kWrong;
    int4 q = make_int4(0, 0, 0, 0);
    if (ok) {
        q = *(const int4*)s_given[x.w];
        flags = copies(p, x) ? kTakes : 0;
        if (flags)
            p.from[seg] = make_int2(p.table[((int64_t)(g * p.W + x.parent) * p.layers + l) * p.max_pages + (x.new_len >> p.shift)],
                                    x.new_len & ((1 << p.shift) - 1));
    }
    ((uint8_t*)p.flags)[seg] = (uint8_t)flags;
    ((int*)p.given)[seg] = q.x + q.y + q.z + q.w;
    p.quarters[seg] = q;
}

struct Sums { int bad, taken, given; };
// 0: done
__device__ __forceinline__ int verdict(const ReorderParams& p, const int4& hd, const Sums& all) {
    if (all.bad || ring_range(hd.x, hd.y, all.given, p.num_pages)) return PKV_PAGES_RANGE;
    return all.taken > hd.y ? PKV_PAGES_SHORT : 0;
}

__device__ __forceinline__ int2 scanned(int2 x, int lane) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int ux = __shfl_up(x.x, d, kWave), uy = __shfl_up(x.y, d, kWave);
        if (lane >= d) { x.x += ux; x.y += uy; }
    }
    return x;
}
__device__ __forceinline__ int2 of_four(uint32_t f, const int4& g) { return make_int2(__popc(f & 0x01010101u), g.x + g.y + g.z + g.w); }

__global__ void __launch_bounds__(kSumThreads)
reorder_sums_kernel(ReorderParams p) {
    __shared__ int2 s_sum[kSumThreads / kWave];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    if (tid == 0) s_bad = 0;
    int2 carry = make_int2(0, 0);
    uint32_t bad = 0;
    for (int base = 0; base < p.n; base += 4 * kSumThreads) {
        const int i = base + 4 * tid;
        uint32_t f = 0;
        int4 g = make_int4(0, 0, 0, 0);
        if (i < p.n) { f = p.flags[i / 4]; g = p.given[i / 4]; }
        bad |= f & (0x01010101u * kWrong);
        const int2 mine = of_four(f, g), incl = scanned(mine, lane);
        __syncthreads();                                            // (the round before has read its sums)
        if (lane == kWave - 1) s_sum[wv] = incl;
        __syncthreads();
        int2 before = make_int2(carry.x + incl.x - mine.x, carry.y + incl.y - mine.y);
        for (int w = 0; w < kSumThreads / kWave; ++w) {
            const int2 y = s_sum[w];
            if (w < wv) { before.x += y.x; before.y += y.y; }
            carry.x += y.x; carry.y += y.y;
        }
        const int ge[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e < p.n) p.first[i + e] = before;
            before.x += (f >> (8 * e)) & 1u;
            before.y += ge[e];
        }
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (tid == 0) {
        const int4 hd = p.head[0];
        const int status = verdict(p, hd, Sums{s_bad, carry.x, carry.y});
        p.head[0] = make_int4(hd.x, hd.y, carry.x, carry.y);
        p.head[1] = make_int4(status, 0, 0, 0);
    }
}

// OWN: this workgroup sums up the segments itself.
template <bool OWN>
__global__ void __launch_bounds__(kReorderThreads)
reorder_apply_kernel(ReorderParams p) {
    __shared__ int2 s_sum[kReorderWaves], s_before[kMaxBeams];
    __shared__ uint32_t s_bad[kReorderWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const bool tables = (int)blockIdx.x < p.units;
    int g = 0, l = 0, seg = 0, split = 0;
    int2 from = make_int2(-1, 0);
    const int4 hd = p.head[0];
    GroupPlace x;
    bool known = true;
    if (tables) {
        const DivMod gl = uniform_div_mod((int)blockIdx.x, p.by_layers);
        g = gl.q; l = gl.r;
        known = look(p, g, l, lane, x);
    } else {
        const DivMod ss = uniform_div_mod((int)blockIdx.x - p.units, p.by_splits);
        seg = ss.q; split = ss.r;
        const uint8_t flags = ((const uint8_t*)p.flags)[seg];
        from = p.from[seg];
        if (!(flags & kTakes)) return;                              // nothing to copy
    }
    Sums all;
    int2 before;                                                    // of this segment (tables: of the lane's)
    int status;
    if constexpr (OWN) {
        const int per = (p.n + 4 * kReorderThreads - 1) / (4 * kReorderThreads) * 4, i0 = tid * per;      // segments of a thread
        int2 mine = make_int2(0, 0);
        uint32_t bad = 0;
        for (int i = i0; i < min(i0 + per, p.n); i += 4) {
            const uint32_t f = p.flags[i / 4];
            const int2 y = of_four(f, p.given[i / 4]);
            bad |= f & (0x01010101u * kWrong);
            mine.x += y.x; mine.y += y.y;
        }
        const int2 incl = scanned(mine, lane);
        const bool wrong = __builtin_amdgcn_ballot_w64(bad != 0) != 0;
        if (lane == kWave - 1) { s_sum[wv] = incl; s_bad[wv] = wrong; }
        __syncthreads();
        int2 start = make_int2(incl.x - mine.x, incl.y - mine.y);
        all = Sums{0, 0, 0};
#pragma unroll
        for (int w = 0; w < kReorderWaves; ++w) {
            const int2 y = s_sum[w];
            if (w < wv) { start.x += y.x; start.y += y.y; }
            all.taken += y.x; all.given += y.y; all.bad |= (int)s_bad[w];
        }
        for (int w = 0; w < (tables ? p.W : 1); ++w) {
            const int at = tables ? (g * p.W + w) * p.layers + l : seg;
            if (at < i0 || at >= i0 + per) continue;
            int2 y = start;
            for (int i = i0; i < at; ++i) { y.x += ((const uint8_t*)p.flags)[i] & kTakes; y.y += ((const int*)p.given)[i]; }
            s_before[w] = y;
        }
        __syncthreads();
        before = s_before[tables ? min(x.w, p.W - 1) : 0];
        status = verdict(p, hd, all);
    } else {
        all = Sums{0, hd.z, hd.w};
        status = p.head[1].x;
        before = p.first[tables ? (int64_t)x.s * p.layers + l : seg];
    }

    if (!tables) {
        if (status != 0) return;
        const int dst = p.ring[ring_place((uint32_t)hd.x + (uint32_t)before.x, p.num_pages)];
        if ((uint32_t)dst >= (uint32_t)p.num_pages || (uint32_t)from.x >= (uint32_t)p.num_pages) return;
        // the used rows of a head lie together: heads h0 ... h1-1, pieces of 16 bytes
        const int h0 = split * p.heads_per, heads = min(p.Hkv - h0, p.heads_per);
        const uint32_t pieces = (uint32_t)from.y << p.row_shift;
        const FastDiv by_pieces = {pieces, 0xffffffffu / pieces};   // (one less than it could be for powers of two: corrected by div_mod)
        const int64_t page = (int64_t)p.row_bytes << p.shift;       // of one head
        const int64_t src = ((int64_t)from.x * p.Hkv + h0) * page, to = ((int64_t)dst * p.Hkv + h0) * page;
        const int all_pieces = heads * (int)pieces;
        constexpr int U = 4;                                        // in flight, of both tensors
        for (int i0 = tid; i0 < all_pieces; i0 += U * kReorderThreads) {
            u32x4_t k[U], v[U];
            int64_t off[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const DivMod x = div_mod(min(i0 + u * kReorderThreads, all_pieces - 1), by_pieces);
                off[u] = x.q * page + 16 * (int64_t)x.r;
                k[u] = *(const u32x4_t*)(p.kp + src + off[u]);
                v[u] = *(const u32x4_t*)(p.vp + src + off[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {                           // (the last piece more than once)
                *(u32x4_t*)(p.kp + to + off[u]) = k[u];
                *(u32x4_t*)(p.vp + to + off[u]) = v[u];
            }
        }
        return;
    }

    if (blockIdx.x == 0 && tid == 0) {
        p.state_out[0] = status ? hd.x : ring_place((uint32_t)hd.x + (uint32_t)all.taken, p.num_pages);
        p.state_out[1] = status ? hd.y : hd.y - all.taken + all.given;
        *p.status = status;
    }
    if (status != 0 || !known) {
        // everything stays: outputs of their own get what there was
        for (int i = wv; i < p.W; i += kReorderWaves) {
            const int64_t row = (int64_t)(g * p.W + i) * p.layers + l;
            const int len = p.lens[row], held = pages_in(p, max(0, min(len, p.max_pages << p.shift)));
            if (p.table_out != p.table)
                for (int j = lane; j < held; j += kWave) p.table_out[row * p.max_pages + j] = p.table[row * p.max_pages + j];
            if (lane == 0) p.lens_out[row] = len;
        }
        return;
    }
    const int4 q = p.quarters[(int64_t)x.s * p.layers + l];
    const bool copied = copies(p, x);
    const int fresh = copied && x.real ? p.ring[ring_place((uint32_t)hd.x + (uint32_t)before.x, p.num_pages)] : -1;
    const Range range = columns_of(p, x, wv);
    if constexpr (!OWN) __syncthreads();                            // (all four have read the lengths)
    if (wv == 0 && x.real && x.col == 0) p.lens_out[(int64_t)x.s * p.layers + l] = x.new_len;
    int to = before.y + (wv > 0 ? q.x : 0) + (wv > 1 ? q.y : 0) + (wv > 2 ? q.z : 0);
    unsigned long long same = 0;                                    // lanes of the place
    for (int c = 0; c < kWave / p.lanes; ++c) same |= 1ull << (x.w + c * p.lanes);
    const unsigned long long lower = same & ((1ull << lane) - 1);   // in the columns before
    int32_t* row = p.table_out + ((int64_t)x.s * p.layers + l) * p.max_pages;
    for (int j0 = range.begin; j0 < range.end; j0 += range.step) {
        const int j = j0 + x.col;
        const Column c = column(p, x, l, lane, j);
        const bool given = c.given && j < range.end;
        const unsigned long long all_given = __builtin_amdgcn_ballot_w64(given);
        if (given)
            p.ring[ring_place((uint32_t)hd.x + (uint32_t)hd.y + (uint32_t)(to + __popcll(all_given & lower)), p.num_pages)] = c.id;
        to += __popcll(all_given & same);
        if (x.real && c.in_new && j < range.end) row[j] = copied && j == x.new_len >> p.shift ? fresh : c.next;
    }
}

// heads that a workgroup copies
static int heads_per_copy(int Hkv, int head_bytes) {
    const int n = kCopyBytes / head_bytes;
    return n < 1 ? 1 : n < Hkv ? n : Hkv;
}

// workgroups are counted in 24 bits, as a grid's threads (256 of a workgroup) are in 32
bool reorder_fits(int S, int W, int Hkv, int row_bytes, const pkv_paging& g) {
    const int per = heads_per_copy(Hkv, g.page_size * row_bytes);
    return (int64_t)S / W * g.layers + (int64_t)S * g.layers * ((Hkv + per - 1) / per) < 1 << 24;
}

static size_t in_fours(int S, int layers) { return ((size_t)S * layers + 3) / 4 * 4; }
size_t reorder_ws_bytes(int S, int layers) { return 256 + in_fours(S, layers) * (sizeof(int4) + sizeof(int) + 1 + 2 * sizeof(int2)); }

hipError_t launch_reorder(int S, int W, int Hkv, int row_bytes, const pkv_paging& g, const int32_t* parents, const int32_t* table,
                          const int32_t* lens, int32_t* ring, const int32_t* state, int32_t* table_out, int32_t* lens_out,
                          int32_t* state_out, void* kp, void* vp, int32_t* status, void* ws, hipStream_t st) {
    ReorderParams p;
    p.W = W; p.layers = g.layers; p.n = S * g.layers;
    p.lanes = 1;
    while (p.lanes < W) p.lanes *= 2;
    p.num_pages = g.num_pages; p.max_pages = g.max_pages; p.shift = __builtin_ctz((unsigned)g.page_size);
    p.units = S / W * g.layers;
    p.Hkv = Hkv;
    p.heads_per = heads_per_copy(Hkv, g.page_size * row_bytes);
    p.splits = (Hkv + p.heads_per - 1) / p.heads_per;
    p.row_bytes = row_bytes; p.row_shift = __builtin_ctz((unsigned)row_bytes / 16);
    p.by_layers = fast_div(g.layers); p.by_splits = fast_div(p.splits);
    p.parents = parents; p.table = table; p.lens = lens; p.ring = ring; p.state = state;
    p.table_out = table_out; p.lens_out = lens_out; p.state_out = state_out;
    p.kp = (unsigned char*)kp; p.vp = (unsigned char*)vp; p.status = status;
    const size_t n4 = in_fours(S, g.layers);
    p.head = (int4*)ws;
    p.quarters = (int4*)((char*)ws + 256);
    p.given = p.quarters + n4;
    p.from = (int2*)(p.given + n4 / 4);
    p.first = p.from + n4;
    p.flags = (uint32_t*)(p.first + n4);
    // (a single place has nobody to share with: nothing is copied)
    const dim3 grid((unsigned)(p.units + (W > 1 ? p.n * p.splits : 0)));
    hipLaunchKernelGGL(reorder_count_kernel, dim3((unsigned)p.units), dim3(kReorderThreads), 0, st, p);
    if (p.n <= kOwnSums) {
        hipLaunchKernelGGL(reorder_apply_kernel<true>, grid, dim3(kReorderThreads), 0, st, p);
    } else {
        hipLaunchKernelGGL(reorder_sums_kernel, dim3(1), dim3(kSumThreads), 0, st, p);
        hipLaunchKernelGGL(reorder_apply_kernel<false>, grid, dim3(kReorderThreads), 0, st, p);
    }
    return hipGetLastError();
}

}  // namespace pkv
