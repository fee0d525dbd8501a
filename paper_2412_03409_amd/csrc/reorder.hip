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
// Bound: latency for a request's beams, HBM where many partly filled pages are copied.
#include "packed.hpp"
#include "fast_div.hpp"
#include "packed_rules.hpp"

namespace pkv {

constexpr int kReorderThreads = 256;
constexpr int kReorderWaves = kReorderThreads / kWave;
constexpr int kSumThreads = 1024;
constexpr int kOwnSums = 4096;          // segments up to which a workgroup sums them up itself
constexpr int kCopyBytes = 32768;       // of a tensor that a workgroup copies

struct ReorderParams {
    int S, W, layers, n;                // n = S * layers segments
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
    int4* head;                         // workspace: {head, count, taken, given} (the latter two: of all segments), {accepted, status, 0, 0}
    int4* rec;                          // workspace [n]: {taken (-1: a number that cannot be), given, page to copy from, rows}
    int2* first;                        // workspace [n]: sums of both over the segments before
};

// What a lane knows of its place: in every column the same.
struct Place {
    int w, col, s, parent;              // parent: lane of its column, -1
    bool real, again;                   // again: a lower place continues the same one
    int old_len, new_len;
};

__device__ __forceinline__ int pages_in(const ReorderParams& p, int len) { return (len + (1 << p.shift) - 1) >> p.shift; }

// -> false where a parent or a length cannot be (of the whole group's)
__device__ __forceinline__ bool look(const ReorderParams& p, int g, int l, int lane, Place& x) {
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
__device__ __forceinline__ bool copies(const ReorderParams& p, const Place& x) { return x.again && (x.new_len & ((1 << p.shift) - 1)) != 0; }

struct Column { int id, next; bool in_old, in_new, given; };     // old and new entry (next: of a copied page the one copied from)
__device__ __forceinline__ Column column(const ReorderParams& p, const Place& x, int l, int lane, int j) {
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
__device__ __forceinline__ Range columns_of(const ReorderParams& p, const Place& x, int wv) {
    int most = max(pages_in(p, x.old_len), pages_in(p, x.new_len));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = max(most, __shfl_xor(most, d, kWave));
    const int step = kWave / p.lanes, each = (most + kReorderWaves * step - 1) / (kReorderWaves * step) * step;
    return {min(most, wv * each), min(most, (wv + 1) * each), step};
}
// pages that this wavefront's columns give back, of each place (in the lanes of column 0)
__device__ __forceinline__ int count_given(const ReorderParams& p, const Place& x, int l, int lane, const Range& r) {
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
    __shared__ int s_given[kReorderWaves][kMaxBeams];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const DivMod gl = uniform_div_mod((int)blockIdx.x, p.by_layers);
    const int g = gl.q, l = gl.r;
    if (blockIdx.x == 0 && tid == 0) p.head[0] = make_int4(p.state[0], p.state[1], 0, 0);
    Place x;
    const bool ok = look(p, g, l, lane, x);
    if (ok) {
        const int given = count_given(p, x, l, lane, columns_of(p, x, wv));
        if (x.real && x.col == 0) s_given[wv][x.w] = given;
    }
    __syncthreads();
    if (wv != 0 || !x.real || x.col != 0) return;
    int4 r = make_int4(-1, 0, -1, 0);
    if (ok) {
        r.y = 0;
#pragma unroll
        for (int i = 0; i < kReorderWaves; ++i) r.y += s_given[i][x.w];
        r.x = copies(p, x) ? 1 : 0;
        if (r.x) {
            r.z = p.table[((int64_t)(g * p.W + x.parent) * p.layers + l) * p.max_pages + (x.new_len >> p.shift)];
            r.w = x.new_len & ((1 << p.shift) - 1);
        }
    }
    p.rec[(int64_t)x.s * p.layers + l] = r;
}

struct Sums { int bad, taken, given; };
// 0: done
__device__ __forceinline__ int verdict(const ReorderParams& p, const int4& hd, const Sums& all) {
    if (all.bad || ring_range(hd.x, hd.y, all.given, p.num_pages)) return PKV_PAGES_RANGE;
    return all.taken > hd.y ? PKV_PAGES_SHORT : 0;
}

__global__ void __launch_bounds__(kSumThreads)
reorder_sums_kernel(ReorderParams p) {
    __shared__ int2 s_sum[kSumThreads / kWave];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    if (tid == 0) s_bad = 0;
    int2 carry = make_int2(0, 0);
    bool bad = false;
    for (int base = 0; base < p.n; base += kSumThreads) {
        const int i = base + tid;
        int2 mine = make_int2(0, 0);
        if (i < p.n) {
            const int4 r = p.rec[i];
            bad = bad || r.x < 0;
            mine = make_int2(max(r.x, 0), r.y);
        }
        int2 incl = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int ux = __shfl_up(incl.x, d, kWave), uy = __shfl_up(incl.y, d, kWave);
            if (lane >= d) { incl.x += ux; incl.y += uy; }
        }
        __syncthreads();                                        // (the round before has read its sums)
        if (lane == kWave - 1) s_sum[wv] = incl;
        __syncthreads();
        int2 before = make_int2(carry.x + incl.x - mine.x, carry.y + incl.y - mine.y);
        for (int w = 0; w < kSumThreads / kWave; ++w) {
            const int2 y = s_sum[w];
            if (w < wv) { before.x += y.x; before.y += y.y; }
            carry.x += y.x; carry.y += y.y;
        }
        if (i < p.n) p.first[i] = before;
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
    __shared__ int s_row[kMaxBeams][2], s_part[kMaxBeams][2];       // a place's layers, those in front of this one
    __shared__ int s_sum[5], s_given[kReorderWaves][kMaxBeams];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const bool tables = (int)blockIdx.x < p.units;
    int g, l, seg = 0, split = 0;
    int4 r = make_int4(0, 0, -1, 0);
    if (tables) {
        const DivMod gl = uniform_div_mod((int)blockIdx.x, p.by_layers);
        g = gl.q; l = gl.r;
    } else {
        const DivMod ss = uniform_div_mod((int)blockIdx.x - p.units, p.by_splits);
        seg = ss.q; split = ss.r;
        r = p.rec[seg];
        if (r.x <= 0) return;                                       // nothing to copy
        const DivMod sl = uniform_div_mod(seg, p.by_layers);
        g = sl.q / p.W; l = sl.r;
    }
    const int4 hd = p.head[0];
    Sums all;
    int2 before = make_int2(0, 0);                                  // of this place's segment (tables: of lane's)
    int status;
    const int w = tables ? lane & (p.lanes - 1) : seg / p.layers - g * p.W;
    if constexpr (OWN) {
        for (int i = tid; i < kMaxBeams * 2; i += kReorderThreads) { (&s_row[0][0])[i] = 0; (&s_part[0][0])[i] = 0; }
        if (tid < 5) s_sum[tid] = 0;
        __syncthreads();
        const int from = g * p.W * p.layers, to = from + p.W * p.layers;
        int bad = 0, tx = 0, ty = 0, bx = 0, by = 0;
        for (int i = tid; i < p.n; i += kReorderThreads) {
            const int2 y = *(const int2*)(p.rec + i);
            const int taken = max(y.x, 0);
            bad |= y.x < 0;
            tx += taken; ty += y.y;
            if (i < from) { bx += taken; by += y.y; }
            else if (i < to && (taken | y.y) != 0) {
                const DivMod sl = div_mod(i - from, p.by_layers);
                atomicAdd(&s_row[sl.q][0], taken);
                atomicAdd(&s_row[sl.q][1], y.y);
                if (sl.r < l) { atomicAdd(&s_part[sl.q][0], taken); atomicAdd(&s_part[sl.q][1], y.y); }
            }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            bad |= __shfl_xor(bad, d, kWave);
            tx += __shfl_xor(tx, d, kWave); ty += __shfl_xor(ty, d, kWave);
            bx += __shfl_xor(bx, d, kWave); by += __shfl_xor(by, d, kWave);
        }
        if (lane == 0) {
            if (bad) atomicOr(&s_sum[0], 1);
            atomicAdd(&s_sum[1], tx); atomicAdd(&s_sum[2], ty);
            atomicAdd(&s_sum[3], bx); atomicAdd(&s_sum[4], by);
        }
        __syncthreads();
        all = Sums{s_sum[0], s_sum[1], s_sum[2]};
        before = make_int2(s_sum[3], s_sum[4]);
        for (int i = 0; i < min(w, p.W); ++i) { before.x += s_row[i][0]; before.y += s_row[i][1]; }
        if (w < p.W) { before.x += s_part[w][0]; before.y += s_part[w][1]; }
        status = verdict(p, hd, all);
    } else {
        all = Sums{0, hd.z, hd.w};
        status = p.head[1].x;
        before = p.first[tables ? (int64_t)(g * p.W + min(w, p.W - 1)) * p.layers + l : seg];
    }

    if (!tables) {
        if (status != 0) return;
        const int dst = p.ring[ring_place((uint32_t)hd.x + (uint32_t)before.x, p.num_pages)];
        if ((uint32_t)dst >= (uint32_t)p.num_pages || (uint32_t)r.z >= (uint32_t)p.num_pages) return;
        // the used rows of a head lie together: heads h0 ... h1-1, pieces of 16 bytes
        const int h0 = split * p.heads_per, heads = min(p.Hkv - h0, p.heads_per);
        const uint32_t pieces = (uint32_t)r.w << p.row_shift;       // (above 1)
        const FastDiv by_pieces = {pieces, (uint32_t)((1ull << 32) / pieces)};
        const int64_t page = (int64_t)p.row_bytes << p.shift;       // of one head
        const int64_t src = ((int64_t)r.z * p.Hkv + h0) * page, to = ((int64_t)dst * p.Hkv + h0) * page;
        const int all_pieces = heads * (int)pieces;
        constexpr int U = 4;                                        // in flight, of both tensors
        for (int i0 = tid; i0 < all_pieces; i0 += U * kReorderThreads) {
            uint4 k[U], v[U];
            int64_t off[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const DivMod x = div_mod(min(i0 + u * kReorderThreads, all_pieces - 1), by_pieces);
                off[u] = x.q * page + 16 * (int64_t)x.r;
                k[u] = *(const uint4*)(p.kp + src + off[u]);
                v[u] = *(const uint4*)(p.vp + src + off[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * kReorderThreads < all_pieces) {
                    *(uint4*)(p.kp + to + off[u]) = k[u];
                    *(uint4*)(p.vp + to + off[u]) = v[u];
                }
        }
        return;
    }

    if (blockIdx.x == 0 && tid == 0) {
        p.state_out[0] = status ? hd.x : ring_place((uint32_t)hd.x + (uint32_t)all.taken, p.num_pages);
        p.state_out[1] = status ? hd.y : hd.y - all.taken + all.given;
        *p.status = status;
    }
    if (status != 0) {
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
    Place x;
    look(p, g, l, lane, x);
    const Range range = columns_of(p, x, wv);
    const int mine = count_given(p, x, l, lane, range);
    if (x.real && x.col == 0) s_given[wv][x.w] = mine;
    __syncthreads();                                                // (all four have read the lengths)
    if (wv == 0 && x.real && x.col == 0) p.lens_out[(int64_t)x.s * p.layers + l] = x.new_len;
    int to = before.y;
    for (int i = 0; i < wv; ++i) to += s_given[i][min(x.w, p.W - 1)];
    const bool copied = copies(p, x);
    const int fresh = copied && x.real ? p.ring[ring_place((uint32_t)hd.x + (uint32_t)before.x, p.num_pages)] : -1;
    unsigned long long lower = 0;                                   // lanes of the place in the columns before
    for (int c = 0; c < x.col; ++c) lower |= 1ull << (x.w + c * p.lanes);
    unsigned long long same = 0;
    for (int c = 0; c < kWave / p.lanes; ++c) same |= 1ull << (x.w + c * p.lanes);
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

size_t reorder_ws_bytes(int S, int layers) { return 256 + (size_t)S * layers * (sizeof(int4) + sizeof(int2)); }

hipError_t launch_reorder(int S, int W, int Hkv, int row_bytes, const pkv_paging& g, const int32_t* parents, const int32_t* table,
                          const int32_t* lens, int32_t* ring, const int32_t* state, int32_t* table_out, int32_t* lens_out,
                          int32_t* state_out, void* kp, void* vp, int32_t* status, void* ws, hipStream_t st) {
    ReorderParams p;
    p.S = S; p.W = W; p.layers = g.layers; p.n = S * g.layers;
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
    p.head = (int4*)ws; p.rec = (int4*)((char*)ws + 256); p.first = (int2*)(p.rec + p.n);
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
