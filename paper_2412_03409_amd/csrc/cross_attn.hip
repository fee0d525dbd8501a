// Attention of many bf16 rows to states of another length: every row of a sequence sees all of its states, or the first seen[t] of them.
// Query heads that share a KV head are rows of one tile, row = token * heads + head.
//
//  cross_tiles_kernel  A workgroup has 128 rows of one (sequence, KV head) and a piece of the states, which stream through LDS 64 at a
//                      time (asynchronous copies, two buffer pairs); a wavefront has 32 rows.  Bound: the matrix cores and the softmax
//                      next to them.  Two texts of up to 4001 rows over up to 6001 states, H32/8: 444 GFLOP in 455 ... 490 us.
//  cross_merge_kernel  joins the pieces of a tile.  Bound: HBM, 66 KB of a part, and the launch: 5 ... 10 us.
//
// How long the sequences and their states are is known on the device only, and a launch of a workgroup per tile takes as long as its
// longest one.  So every workgroup adds up the stages of all tiles, one lane per sequence, and takes the same cap: no piece has more than
// a kPieces-th of all stages (kLeastStages at least).  Then there are kPieces pieces more than tiles at most, which bounds the grid, and at most
// 2 kPieces of tiles that are cut, which bounds the workspace.  Rows that see the first states only leave such a plan uneven: where the work
// is large, a launch of its own (cross_plan_kernel, 6 to 7 us) looks at what each tile sees first, gives its pieces that length, and begins with the longest.
// 6 texts of up to 700 rows over up to 2885 states, H32/8, 13.7 GFLOP: 6.5 + 32 + 8.5 us (without 49 + 10).
//
// Probabilities are rounded to bf16 for the second product, against the running maximum, as for prompts (attn_tile.hpp): with twice the
// second products they would hold 16 bits, which matrix cores that bound the kernel have no room for.  The outputs are 0.0004 to 0.0013 from those of 32-bit
// probabilities, relative over all elements, and 0.0014 to 0.0017 from 64 bits, as those are: most of it is their own rounding to bf16.
//
// Stages that some rows see and others do not are masked, and a probability of 0 times an infinite or NaN value that such a row must not
// see would spoil it.  To look for such values in every masked stage costs a third of it, so a tile is worked on without, and again with
// the look if a row of it came out infinite or NaN.
#include "attn_tile.hpp"

#include <type_traits>

namespace pkv {

struct CrossParams {
    int S, T, M, grp, max_rows;
    int heads, heads_per_xcd;           // heads: L * Hkv; heads_per_xcd: 0 if they do not divide up
    FastDiv by_grp, by_hkv, by_heads;
    const unsigned char *q, *k, *v;
    unsigned char* out;
    Strides qs, ks, vs, os;             // in bytes
    const int32_t *row_off, *state_off, *seen;
    const float* scale;
    float* part_o;                      // workspace [2 * kPieces][4 wavefronts][32 * D], as registers are
    float2* part_ms;                    // [2 * kPieces][4 wavefronts][64]: {maximum, sum}; sum 0: nothing seen, no numerators
    int4* planned;                      // {places, pieces of cut tiles, cut tiles, 0} of a head, then two a place, then two a cut tile
};
// (320, 384, 512, 768, 1024 pieces: 21.9, 21.8, 22.3, 22.8, 23.3 us, the geometric mean of 70 calls of all sizes; at least 8 stages a piece: 22.2)
constexpr int kPieces = 384;
constexpr int kLeastStages = 4;
constexpr int kManyTiles = 2048;        // from which on no tile is cut

struct Text { int s, first, rows, from, len; };     // rows: of the call, times the heads of a KV head; from, len: its states
__device__ __forceinline__ Text text_of(const CrossParams& p, int s) {
    const int first = p.row_off[s], last = p.row_off[s + 1], from = p.state_off[s], to = p.state_off[s + 1];
    return {s, first, min(new_rows(first, last, p.T), p.max_rows) * p.grp, from, new_rows(from, to, p.M)};
}
__device__ __forceinline__ int tiles_of(const Text& x) { return (x.rows + kTileRows - 1) / kTileRows; }
__device__ __forceinline__ int stages_of(const Text& x) { return (x.len + kStage - 1) / kStage; }
__device__ __forceinline__ int pieces_of(const Text& x, int cap) { return x.rows == 0 ? 0 : max(1, (stages_of(x) + cap - 1) / cap); }

// The texts of a head, one per lane (beyond 64 they are read again): the cap on a piece, and the places of a head, which are the pieces of
// all tiles or (MERGE) the tiles that are cut.
template <bool MERGE, bool CUT>
struct Plan {
    const CrossParams& p;
    int lane, cap;
    Text mine;
    int upto, cut_upto;                 // places of the first 64 texts up to this lane's; pieces of cut tiles
    int places, cuts;                   // of all (below 2^24; 2 kPieces)

    __device__ __forceinline__ Plan(const CrossParams& params, int ln) : p(params), lane(ln) {
        mine = text_of(p, min(lane, p.S - 1));
        cap = 1 << 30;
        if constexpr (CUT) {
            int64_t all = lane < p.S ? (int64_t)tiles_of(mine) * stages_of(mine) : 0;
            for (int s = lane + kWave; s < p.S; s += kWave) {
                const Text x = text_of(p, s);
                all += (int64_t)tiles_of(x) * stages_of(x);
            }
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) {
                const int lo = __shfl_xor((int)(uint32_t)all, d, kWave), hi = __shfl_xor((int)(all >> 32), d, kWave);
                all += (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
            }
            cap = __builtin_amdgcn_readfirstlane(max(kLeastStages, (int)fmin((double)all * p.heads / kPieces, 1e9) + 1));
        }
        places = cuts = 0;
        for (int s0 = 0; s0 < p.S; s0 += kWave) {
            int a, b;
            scan(s0, s0 == 0 ? mine : text_of(p, min(s0 + lane, p.S - 1)), a, b);
            if (s0 == 0) { upto = a; cut_upto = b; }
            const int last = min(p.S - s0, kWave) - 1;
            places += __builtin_amdgcn_readlane(a, last);
            cuts += __builtin_amdgcn_readlane(b, last);
        }
    }
    __device__ __forceinline__ int size(const Text& x) const {
        if constexpr (!CUT) return tiles_of(x);
        const int pieces = pieces_of(x, cap);
        return MERGE ? (pieces > 1 ? tiles_of(x) : 0) : pieces * tiles_of(x);
    }
    __device__ __forceinline__ int cut_size(const Text& x) const {
        if constexpr (!CUT) return 0;
        const int pieces = pieces_of(x, cap);
        return pieces > 1 ? pieces * tiles_of(x) : 0;
    }
    // sums over the texts s0 ... s0 + lane
    __device__ __forceinline__ void scan(int s0, const Text& x, int& a, int& b) const {
        const bool real = s0 + lane < p.S;
        a = real ? size(x) : 0;
        b = real ? cut_size(x) : 0;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            if (d >= p.S) break;
            const int ua = __shfl_up(a, d, kWave), ub = CUT ? __shfl_up(b, d, kWave) : 0;
            if (lane >= d) { a += ua; b += ub; }
        }
    }
    // the text that holds place x (below `places`), the place in it, and the pieces of cut tiles before it
    __device__ __forceinline__ Text find(int x, int& in, int& cut_before) const {
        int s0 = 0, base = 0, cut = 0, a = upto, b = cut_upto;
        Text y = mine;
        while (s0 + kWave < p.S && __builtin_amdgcn_ballot_w64(base + a > x) == 0) {
            base += __builtin_amdgcn_readlane(a, kWave - 1);
            cut += __builtin_amdgcn_readlane(b, kWave - 1);
            s0 += kWave;
            y = text_of(p, min(s0 + lane, p.S - 1));
            scan(s0, y, a, b);
        }
        const unsigned long long at = __builtin_amdgcn_ballot_w64(s0 + lane < p.S && base + a > x);
        Text t = {0, 0, 0, 0, 0};
        in = cut_before = 0;
        if (at == 0) return t;                                  // (offsets that descend may add up to more places than there are numbers)
        const int j = __builtin_ctzll(at);
        t.s = s0 + j;
        t.first = __builtin_amdgcn_readlane(y.first, j); t.rows = __builtin_amdgcn_readlane(y.rows, j);
        t.from = __builtin_amdgcn_readlane(y.from, j); t.len = __builtin_amdgcn_readlane(y.len, j);
        in = x - base - __builtin_amdgcn_readlane(a, j) + size(t);
        cut_before = cut + __builtin_amdgcn_readlane(b, j) - cut_size(t);
        return t;
    }
};

// how many of its text's states row `row` of it sees
__device__ __forceinline__ int seen_by(const CrossParams& p, const Text& x, int row) {
    return max(0, min(p.seen[x.first + row_at(row, p.by_grp).token], x.len));
}
// Limits of the rows row0 ... row0+ROWS-1
template <int ROWS>
__device__ __forceinline__ Limits limits(const CrossParams& p, const Text& x, int row0, int lane) {
    int lo = x.len, hi = 0;
#pragma unroll
    for (int i = 0; i < (ROWS + kWave - 1) / kWave; ++i) {
        const int n = seen_by(p, x, min(row0 + min(i * kWave + lane, ROWS - 1), x.rows - 1));
        lo = min(lo, n);
        hi = max(hi, n);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        lo = min(lo, __shfl_xor(lo, d, kWave));
        hi = max(hi, __shfl_xor(hi, d, kWave));
    }
    return {__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi)};
}

// The same plan where rows see the first states only, by what some row of each tile sees: written out, a list of places and one of cut tiles.
struct Place { Text text; int tile, pieces, piece, slot, end, all; };       // slot: of the tile's first part; end, all: states that some, and all of its rows see
constexpr int kPlanThreads = 1024;      // texts at most
constexpr int kPlaces = kManyTiles + kPieces;
constexpr size_t kPlanBytes = (1 + 2 * (kPlaces + kPieces)) * sizeof(int4);
static_assert(kPieces < 512 && kManyTiles == 2 * kPlanThreads, "nine bits in a place; two tiles a thread");
__device__ __forceinline__ void write_place(int4* to, const Place& x) {
    to[0] = make_int4(x.text.first, x.text.rows, x.text.from, x.text.len);
    to[1] = make_int4(x.tile, x.pieces | x.piece << 9 | x.slot << 18, x.end, x.all);
}
__device__ __forceinline__ Place read_place(const int4* from) {
    const int4 a = from[0], b = from[1];
    return {{0, a.x, a.y, a.z, a.w}, b.x, b.y & 511, b.y >> 9 & 511, b.y >> 18, b.z, b.w};
}
// sums of x over the threads 0 ... threadIdx.x, and of all
template <typename T>
__device__ __forceinline__ T block_sums(T x, T* cells, T& all) {
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const T up = __shfl_up(x, d, kWave);
        if (lane >= d) x += up;
    }
    if (lane == kWave - 1) cells[wv] = x;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / kWave; ++w) {
        if (w < wv) before += cells[w];
        all += cells[w];
    }
    return before + x;
}
__global__ void __launch_bounds__(kPlanThreads)
cross_plan_kernel(CrossParams p) {
    constexpr int kGroup = 16;          // lanes that look at a tile's rows
    constexpr int kLengths = 16;        // classes of pieces, the longest first
    __shared__ Text s_text[kPlanThreads];
    __shared__ int s_upto[kPlanThreads], s_at[kManyTiles], s_end[kManyTiles], s_all[kManyTiles];
    __shared__ int s_tiles[kPlanThreads / kWave];
    __shared__ double s_work[kPlanThreads / kWave];
    __shared__ uint32_t s_sums[kPlanThreads / kWave];
    __shared__ int s_length[kLengths], s_next[kLengths];
    const int tid = threadIdx.x;
    if (tid < kLengths) s_length[tid] = s_next[tid] = 0;
    int tiles = 0;
    if (tid < p.S) {
        s_text[tid] = text_of(p, tid);
        tiles = tiles_of(s_text[tid]);
    }
    int all;
    s_upto[tid] = block_sums(tiles, s_tiles, all);
    all = min(all, kManyTiles);                                 // (more only where texts overlap)
    __syncthreads();
    for (int i = tid / kGroup; i < all; i += kPlanThreads / kGroup) {
        int s = 0, behind = p.S - 1;                            // the first text whose sum is above i
        while (s < behind) {
            const int mid = (s + behind) / 2;
            if (s_upto[mid] > i) behind = mid;
            else s = mid + 1;
        }
        const Text t = s_text[s];
        const int tile = i - (s == 0 ? 0 : s_upto[s - 1]), r0 = tile * kTileRows;
        const int from = row_at(r0, p.by_grp).token, to = row_at(min(r0 + kTileRows, t.rows) - 1, p.by_grp).token;
        int lo = t.len, hi = 0;
#pragma unroll 4
        for (int k = from + tid % kGroup; k <= to; k += kGroup) {
            const int n = max(0, min(p.seen[t.first + k], t.len));
            lo = min(lo, n);
            hi = max(hi, n);
        }
#pragma unroll
        for (int d = kGroup / 2; d > 0; d >>= 1) {
            lo = min(lo, __shfl_xor(lo, d, kWave));
            hi = max(hi, __shfl_xor(hi, d, kWave));
        }
        if (tid % kGroup == 0) {
            s_at[i] = s;
            s_end[i] = hi;
            s_all[i] = lo;
        }
    }
    __syncthreads();
    int stages[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) stages[k] = 2 * tid + k < all ? (s_end[2 * tid + k] + kStage - 1) / kStage : 0;
    double work;
    block_sums((double)stages[0] + (double)stages[1], s_work, work);
    const int cap = max(kLeastStages, (int)fmin(work * p.heads / kPieces, 1e9) + 1);
    // pieces of cut tiles and cut tiles in one sum; all pieces by their length, so that a launch does not end with its longest
    uint32_t n[2];
    int pieces[2], length[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        pieces[k] = 2 * tid + k < all ? max(1, (stages[k] + cap - 1) / cap) : 0;
        n[k] = pieces[k] > 1 ? (uint32_t)pieces[k] | 1u << 16 : 0u;
        const int most = pieces[k] > 1 ? (stages[k] + pieces[k] - 1) / pieces[k] : stages[k];
        length[k] = most == 0 ? kLengths - 1 : kLengths - 2 - (int)((float)most * (kLengths - 1) / ((float)cap + 1.f));
        if (pieces[k] > 0) atomicAdd(&s_length[length[k]], pieces[k]);
    }
    uint32_t sums, before = block_sums(n[0] + n[1], s_sums, sums) - n[0] - n[1];
    int upto[kLengths], places = 0;
#pragma unroll
    for (int c = 0; c < kLengths; ++c) {
        upto[c] = places;
        places += s_length[c];
    }
    if (tid == 0) p.planned[0] = make_int4(places, (int)(sums & 0xffff), (int)(sums >> 16), 0);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (pieces[k] == 0) break;
        const int i = 2 * tid + k, s = s_at[i];
        Place x = {s_text[s], i - (s == 0 ? 0 : s_upto[s - 1]), pieces[k], 0, (int)(before & 0xffff), s_end[i], s_all[i]};
        int first = 0;
#pragma unroll
        for (int c = 0; c < kLengths; ++c) first = c == length[k] ? upto[c] : first;
        int4* to = p.planned + 1 + 2 * (first + atomicAdd(&s_next[length[k]], pieces[k]));
        if (pieces[k] > 1) write_place(p.planned + 1 + 2 * (kPlaces + (int)(before >> 16)), x);
        for (; x.piece < x.pieces; ++x.piece, to += 2) write_place(to, x);
        before += n[k];
    }
}

// SEEN: rows see the first states only.  CUT: tiles may be cut.  PLANNED: as cross_plan_kernel says.
template <int D, bool SEEN, bool CUT, bool PLANNED>
__global__ void __launch_bounds__(256, 2)
cross_tiles_kernel(CrossParams p) {
    constexpr int ROWB = D * 2, kInst = CopyLane<D>::kCopies;               // copies per wavefront, stage and tensor: 16 rows
    __shared__ __attribute__((aligned(1024))) unsigned char sKa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sKb[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVb[kStage * ROWB];
    __shared__ int s_wild;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int ln = lane & 31, hf = lane >> 5;
    if (SEEN && threadIdx.x == 0) s_wild = 0;

    // Which tile and piece.  With heads in eighths every head stays on one XCD, else they alternate; in a head text by text, the tiles of
    // a piece of the states one after the other, so that they are read through the same L2 at about the same time.
    int head, x;
    auto place = [&](int places) {                                          // whether there is one
        if (places <= 0) return false;
        if (p.heads_per_xcd > 0) {
            const uint32_t j = blockIdx.x / kXcds, h = j / (uint32_t)places;
            head = (int)(blockIdx.x % kXcds) * p.heads_per_xcd + (int)h;
            x = (int)(j - h * (uint32_t)places);
            return h < (uint32_t)p.heads_per_xcd;
        }
        const DivMod hx = uniform_div_mod((int)blockIdx.x, p.by_heads);
        head = hx.r; x = hx.q;
        return hx.q < places;
    };
    Place at;
    int cuts = 0;
    if constexpr (PLANNED) {
        const int4 sums = p.planned[0];
        if (!place(sums.x)) return;
        cuts = sums.y;
        at = read_place(p.planned + 1 + 2 * x);
    } else {
        const Plan<false, CUT> plan(p, lane);
        if (!place(plan.places)) return;
        int in, cut_before;
        at.text = plan.find(x, in, cut_before);
        if (at.text.rows == 0) return;
        const int tiles = tiles_of(at.text);
        at.pieces = CUT ? pieces_of(at.text, plan.cap) : 1;
        at.piece = CUT ? __builtin_amdgcn_readfirstlane((uint32_t)in / (uint32_t)tiles) : 0;
        at.tile = in - at.piece * tiles;
        at.slot = cut_before + at.tile * at.pieces;
        cuts = plan.cuts;
        at.end = at.all = at.text.len;
        if constexpr (SEEN) {
            const Limits tl = limits<kTileRows>(p, at.text, at.tile * kTileRows, lane);
            at.end = tl.some; at.all = tl.all;
        }
    }
    const Text t = at.text;
    const int tile = at.tile, pieces = at.pieces, piece = at.piece, end = at.end, all = at.all, ends = (end + kStage - 1) / kStage;
    const int stages = PLANNED ? ends : stages_of(t);
    const DivMod lg = uniform_div_mod(head, p.by_hkv);                      // layer, KV head
    const int st0 = CUT ? piece * stages / pieces : 0, st1 = CUT ? min((piece + 1) * stages / pieces, ends) : ends;

    // this wavefront's rows (those that do not exist repeat one that does)
    const int r0 = tile * kTileRows + wv * 32, row = r0 + ln;
    const bool mine = r0 < t.rows, real = row < t.rows;
    const int rr = real ? row : mine ? r0 : 0;
    const RowAt ra = row_at(rr, p.by_grp);
    int lim = t.len - 1, lim_first = lim, lim_last = lim;                   // the last state that the row sees, and the wavefront's rows
    if constexpr (SEEN) {
        const Limits w = limits<32>(p, t, mine ? r0 : 0, lane);
        lim = seen_by(p, t, rr) - 1;
        lim_first = w.all - 1; lim_last = w.some - 1;
    }
    const int n = max(0, st1 - st0), plain = max(0, min(st1, all / kStage) - st0);

    const unsigned char* kb = p.k + p.ks.l * lg.q + p.ks.h * lg.r + p.ks.n * (int64_t)t.from;
    const unsigned char* vb = p.v + p.vs.l * lg.q + p.vs.h * lg.r + p.vs.n * (int64_t)t.from;
    const CopyLane<D> cp(lane);
    auto issue = [&](int st, unsigned char* dK, unsigned char* dV) {        // a wavefront copies 16 rows of each
        const int key = min(st * kStage + wv * 16, end - 1);                // the group's first state, or the last one there is
        const uint32_t rest = (uint32_t)(end - 1 - key);
        const unsigned char *ka = kb + p.ks.n * (int64_t)key, *va = vb + p.vs.n * (int64_t)key;
#pragma unroll
        for (int i = 0; i < kInst; ++i) {
            copy_to_lds(ka + cp.at(i, rest, (uint32_t)p.ks.n), dK + (wv * kInst + i) * 1024);
            copy_to_lds(va + cp.at(i, rest, (uint32_t)p.vs.n), dV + (wv * kInst + i) * 1024);
        }
    };
    auto sync = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wavefront's part of the stage has landed
        __syncthreads();                                     // ... and everybody's; the other pair is free again
    };
    // The last stage is in pair a, so the first one is there if they are odd.
    bool half = (n & 1) != 0;
    if (n > 0) {
        if (half) issue(st0, sKa, sVa);
        else issue(st0, sKb, sVb);
    }
    const float sc = p.scale[lg.q], qs = score_scale(sc);
    const int h = lg.r * p.grp + ra.head;
    const int64_t token = t.first + ra.token;
    RowTile<D> tl;
    tl.offsets(lane);
    tl.load_q(p.q + p.qs.l * lg.q + p.qs.h * h + p.qs.n * token, hf, sc < 0.f);
    tl.clear();

    // Stages that every row of the tile sees, two at a time, without a branch between them.  A wavefront without rows works along on rows
    // that are not stored.
    int st = st0;
    if (half && plain > 0) {
        sync();
        if (st + 1 < st1) issue(st + 1, sKb, sVb);
        tl.template attend<2, false>(sKa, sVa, qs, lane, 0, 0u, 2, 2);
        ++st;
        half = false;
    }
    if (!half) {
        for (; st + 1 < st0 + plain; st += 2) {
            sync();
            issue(st + 1, sKa, sVa);
            tl.template attend<2, false>(sKb, sVb, qs, lane, 0, 0u, 2, 2);
            sync();
            if (st + 2 < st1) issue(st + 2, sKb, sVb);
            tl.template attend<2, false>(sKa, sVa, qs, lane, 0, 0u, 2, 2);
        }
    }
    auto masked = [&](int st, const unsigned char* sK, const unsigned char* sV, auto check) {
        const int key0 = st * kStage;
        if (mine && key0 <= lim_last)
            tl.template attend<2, true, false, decltype(check)::value>(sK, sV, qs, lane, lim - key0, 0u, key0 + 32 <= lim_last ? 2 : 1,
                                                                      (max(lim_first - key0, -1) + 1) / 32);
    };
    // the others: with SEEN any, else the last one behind one that is like those before
    while (st < st1) {
        if (!half) {
            sync();
            issue(st + 1, sKa, sVa);
            if constexpr (SEEN) masked(st, sKb, sVb, std::false_type{});
            else tl.template attend<2, false>(sKb, sVb, qs, lane, 0, 0u, 2, 2);
            ++st;
        }
        half = false;
        sync();
        if (st + 1 < st1) issue(st + 1, sKb, sVb);
        if constexpr (SEEN) masked(st, sKa, sVa, std::false_type{});
        else masked(st, sKa, sVa, std::true_type{});
        ++st;
    }
    if constexpr (SEEN) {
        // 0 times what is infinite or NaN is NaN
        float z = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) z = fmaf(tl.o[dt][r], 0.f, z);
        if (n > plain) {
            if (mine && __builtin_amdgcn_ballot_w64(z != z) != 0) s_wild = 1;
            __syncthreads();
            if (__builtin_expect(s_wild, 0)) {
                tl.clear();
                for (st = st0; st < st1; ++st) {
                    issue(st, sKa, sVa);
                    sync();
                    masked(st, sKa, sVa, std::true_type{});
                    __syncthreads();
                }
            }
        }
    }
    if (!mine) return;
    const float sum = tl.total();
    if (!CUT || pieces == 1) {
        tl.store(p.out + p.os.l * lg.q + p.os.h * h + p.os.n * token, hf, sum == 0.f ? 0.f : 1.f / sum, real);
    } else {
        const int64_t slot = ((int64_t)head * cuts + at.slot + piece) * 4 + wv;
        if (n > 0) tl.store_tile(p.part_o + slot * 32 * D, p.part_ms + slot * kWave, lane, sum);
        else p.part_ms[slot * kWave + lane] = make_float2(-INFINITY, 0.f);
    }
}

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
// Joins the pieces of a tile: a wavefront has 32 columns of 32 rows, in the registers' order, in which the pieces were written.
template <int D, bool PLANNED>
__global__ void __launch_bounds__(256)
cross_merge_kernel(CrossParams p) {
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), dt = (int)blockIdx.y;
    const int ln = lane & 31, hf = lane >> 5;
    int head, cuts;
    Place at;
    if constexpr (PLANNED) {
        const int4 sums = p.planned[0];
        if (sums.z <= 0) return;
        head = __builtin_amdgcn_readfirstlane(blockIdx.x / (uint32_t)sums.z);
        if (head >= p.heads) return;
        cuts = sums.y;
        at = read_place(p.planned + 1 + 2 * (kPlaces + (int)blockIdx.x - head * sums.z));
    } else {
        const Plan<true, true> plan(p, lane);
        if (plan.places <= 0) return;
        head = __builtin_amdgcn_readfirstlane(blockIdx.x / (uint32_t)plan.places);
        if (head >= p.heads) return;
        int cut_before;
        at.text = plan.find((int)blockIdx.x - head * plan.places, at.tile, cut_before);
        if (at.text.rows == 0) return;
        at.pieces = pieces_of(at.text, plan.cap);
        at.slot = cut_before + at.tile * at.pieces;
        cuts = plan.cuts;
    }
    const Text t = at.text;
    const int pieces = at.pieces, r0 = at.tile * kTileRows + wv * 32, row = r0 + ln;
    if (r0 >= t.rows) return;
    const DivMod lg = uniform_div_mod(head, p.by_hkv);
    const float qs = score_scale(p.scale[lg.q]);
    const int64_t first = (int64_t)head * cuts + at.slot;
    float m = -INFINITY, sum = 0.f;
    f32x16_t o;
#pragma unroll
    for (int r = 0; r < 16; ++r) o[r] = 0.f;
    constexpr int U = 4;                                         // pieces that are asked for together
    for (int i0 = 0; i0 < pieces; i0 += U) {                     // a running maximum: every piece is read once
        float2 x[U];
        f32x4_t y[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[u][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if (i0 + u >= pieces) continue;
            const int64_t slot = (first + i0 + u) * 4 + wv;
            x[u] = p.part_ms[slot * kWave + lane];
            const f32x4_t* from = (const f32x4_t*)(p.part_o + slot * 32 * D) + dt * 4 * kWave + lane;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[u][e] = from[e * kWave];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (of a piece that nothing was seen in the numerators were not written)
            const bool any = x[u].y != 0.f;
            const float mx = any ? fmaxf(m, x[u].x) : m, ref = mx == -INFINITY ? 0.f : mx;
            const float c0 = any ? __builtin_amdgcn_exp2f((m - ref) * qs) : 1.f, c1 = __builtin_amdgcn_exp2f((x[u].x - ref) * qs);
            sum = any ? fmaf(sum, c0, x[u].y * c1) : sum;
            m = mx;
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = any ? fmaf(o[e], c0, y[u][e / 4][e % 4] * c1) : o[e];
        }
    }
    const bool real = row < t.rows;
    const RowAt ra = row_at(real ? row : r0, p.by_grp);
    store_columns(o, p.out + p.os.l * lg.q + p.os.h * (lg.r * p.grp + ra.head) + p.os.n * (int64_t)(t.first + ra.token) + 64 * dt, hf,
                  sum == 0.f ? 0.f : 1.f / sum, real);
}

// tiles of all texts and heads, at most
static long long all_tiles(const pkv_packed& s) {
    return ((long long)s.T * (s.H / s.Hkv) / kTileRows + (s.S < s.T ? s.S : s.T)) * s.L * s.Hkv;
}
// Whether tiles may be cut: where texts are long (half as long again as the average is taken for the longest, as lengths are on the device) and
// the tiles would not fill the chip several times over.  Joining costs 4 to 5 us where nothing was cut.  us, whole / cut: H12/4, 14 texts of
// up to 3350 states and 20 rows 71 / 31; H16/8, one of 1827 and 238 rows 39 / 27; H40/40, 3 of up to 186 and 2872 rows 46 / 54; H32/4, 44
// of up to 179 and 5 rows 8.6 / 13; H40/40, 3 of up to 839 and 3909 rows, D 64, 69 / 74 (cut all the same).  One long text among many short ones stays
// whole, H32/8: 150 rows over 5000 states and 31 texts of 40 over 40 95 / 41, 300 over 2500 and 15 of 40 over 30 53 / 39; 700 over 8000 and 31 of 40 over 20 150 / 147.
constexpr double kCutStages = 8.0;
static bool may_cut(const pkv_packed& s, int M) { return 1.5 * M / s.S / kStage > kCutStages && all_tiles(s) < kManyTiles; }

size_t cross_tiles_ws_bytes(const pkv_packed& s, int M) {
    return may_cut(s, M) ? (size_t)2 * kPieces * kTileRows * (s.D * sizeof(float) + 2 * sizeof(float2)) + kPlanBytes : 0;
}

// Whether what the rows see is looked at first.  The launch costs 4 to 6 us; pieces of one length, and the longest first, are worth more where
// the compute units' 512 workgroups have 16 stages each, if rows saw all.  us, without / with: H28/4, 25 rows over 2859 states 26 / 30; 5 texts of up
// to 35 rows over 4377, H12/4, 25 / 31; 6 of up to 700 over 2885, H32/8, 59 / 48; 10 of up to 343 over 7463, H32/4, 88 / 67; of 70 calls, the 33 above: 0.94.
constexpr double kPlanStages = 512 * 16.0;
static bool look_first(const pkv_packed& s, int M) {
    return s.S <= kPlanThreads && (double)all_tiles(s) * M / s.S / kStage >= kPlanStages;
}

template <int D>
static hipError_t launch(const CrossParams& p, long long tiles, bool cut, bool look, hipStream_t st) {
    const dim3 grid((unsigned)(tiles + (cut ? kPieces : 0)));
    auto* kernel = look ? cross_tiles_kernel<D, true, true, true>
                 : cut ? (p.seen ? cross_tiles_kernel<D, true, true, false> : cross_tiles_kernel<D, false, true, false>)
                       : (p.seen ? cross_tiles_kernel<D, true, false, false> : cross_tiles_kernel<D, false, false, false>);
    auto* merge = look ? cross_merge_kernel<D, true> : cross_merge_kernel<D, false>;
    if (look) hipLaunchKernelGGL(cross_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, p);
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, p);
    if (cut) hipLaunchKernelGGL(merge, dim3(kPieces, D / 32), dim3(256), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_cross_tiles(const pkv_packed& s, const PackedAttn& a, hipStream_t st) {
    auto bytes = [](Strides x) { return Strides{0, x.l * 2, x.h * 2, x.n * 2}; };
    CrossParams p;
    p.S = s.S; p.T = s.T; p.M = a.M; p.grp = s.H / s.Hkv; p.max_rows = a.max_rows;
    p.heads = s.L * s.Hkv;
    p.heads_per_xcd = p.heads % kXcds == 0 ? p.heads / kXcds : 0;
    p.by_grp = fast_div(p.grp); p.by_hkv = fast_div(s.Hkv); p.by_heads = fast_div(p.heads);
    p.q = (const unsigned char*)a.q; p.k = (const unsigned char*)a.k; p.v = (const unsigned char*)a.v; p.out = (unsigned char*)a.out;
    p.qs = bytes(a.qs); p.ks = bytes(a.ks); p.vs = bytes(a.vs); p.os = bytes(a.os);
    p.row_off = a.row_off; p.state_off = a.state_off; p.seen = a.seen; p.scale = a.scale;
    p.part_o = (float*)a.ws;
    p.part_ms = (float2*)(p.part_o + (size_t)2 * kPieces * kTileRows * s.D);
    p.planned = (int4*)(p.part_ms + (size_t)2 * kPieces * 4 * kWave);
    const bool cut = may_cut(s, a.M), look = cut && a.seen && look_first(s, a.M);
    return s.D == 128 ? launch<128>(p, all_tiles(s), cut, look, st) : launch<64>(p, all_tiles(s), cut, look, st);
}

}  // namespace pkv
