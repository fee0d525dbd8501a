// The W best continuations of a prompt's W beams: of beam w by token v
//   score(w, v) = scores[w] + x[w,v] - log sum_u exp x[w,u],
// equal ones by ascending w * V + v.  Within a beam the order is that of the logits, so a row's sum and its W largest logits come out
// of one pass, before its log-sum-exp is known; beams meet in a second, small launch.
//
//  beam_scan_kernel   a workgroup has a piece of a row, in registers: its maximum, the sum of its exponentials and its W largest logits.
//                     Which these are: the W-th largest of the threads' maxima is below W logits at least, so only the W threads
//                     that reach it hold candidates, a few more than W on the whole; each finds its rank by counting.
//                     Bound: HBM, one read of the logits.
//  beam_join_kernel   a workgroup has a prompt: log-sum-exp of the rows from their pieces, then the same choice among the pieces'
//                     lists (the W-th largest of their first entries leaves W lists of W entries).
//
// A sum of exponentials of a piece is held in 32 bits (terms of a thread, then a tree); pieces, logarithms and scores in 64, because
// beams are told apart by differences that 32 bits of a score of -10^2 do not hold.
#include "packed.hpp"
#include "fast_div.hpp"

namespace pkv {

constexpr int kScanThreads = 256;
constexpr int kJoinThreads = 256;

struct BeamParams {
    int S, W, V, pieces;            // pieces of a row
    int64_t stride;                 // of a row, in elements
    const void* logits;
    const float* scores;
    const uint8_t* ended;
    int end_token;                  // -1: none
    FastDiv by_pieces;
    int32_t *tokens, *parents;
    float* scores_out;
    uint8_t* ended_out;
    float2* sums;                   // workspace [S*W][pieces]: {maximum, sum}
    float* value;                   // workspace [S*W][pieces][W], descending
    int32_t* token;                 // the same, -1 behind the last
};

// NaN counts as -inf, +inf as the largest finite number, -0 as 0
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e38f) + 0.f; }
// an order-preserving whole number above 0 of a finite value; 0 stands for -inf: no candidate
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x);
    return x == -INFINITY ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    return x == -(double)INFINITY ? 0ull : (u >> 63) ? ~u : u | (1ull << 63);
}

template <class K>
__device__ __forceinline__ K wave_max(K x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) { const K y = __shfl_xor(x, d, kWave); x = y > x ? y : x; }
    return x;
}
template <class K>
__device__ __forceinline__ K wave_min(K x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) { const K y = __shfl_xor(x, d, kWave); x = y < x ? y : x; }
    return x;
}

// The W-th largest of `n` entries in LDS: {key, place}, larger keys first, equal ones by ascending place, key 0: none.  An entry is
// among the W largest if its key is above `key` or equal and its place at most `place`.  Bisection over the keys that there are, by
// counting with ballots: the first key that exactly W reach will do.  Every wavefront does it for itself.
template <class K>
struct Threshold { K key; uint32_t place; };
template <class K>
__device__ __forceinline__ Threshold<K> nth_largest(const K* key, const uint32_t* place, int n, int W, int lane) {
    auto count = [&](auto f) {
        int c = 0;
        for (int i = 0; i < n; i += kWave) c += __popcll(__builtin_amdgcn_ballot_w64(i + lane < n && f(min(i + lane, n - 1))));
        return c;
    };
    K lo = ~(K)0, hi = 0;
    for (int i = lane; i < n; i += kWave) {
        const K k = key[i];
        hi = max(hi, k);
        lo = k != 0 ? min(lo, k) : lo;
    }
    hi = wave_max(hi);
    lo = wave_min(lo);
    if (hi == 0 || count([&](int i) { return key[i] != 0; }) <= W) return {(K)1, ~0u};      // all there are
    while (lo < hi) {                                                    // at least W reach lo, fewer than W pass hi
        const K mid = lo + (hi - lo + 1) / 2;
        const int c = count([&](int i) { return key[i] >= mid; });
        if (c == W) return {mid, ~0u};
        if (c > W) lo = mid; else hi = mid - 1;
    }
    const int above = count([&](int i) { return key[i] > lo; });
    uint32_t a = 0, b = ~0u;                                             // the lowest places of the equal ones
    while (a < b) {
        const uint32_t mid = a + (b - a) / 2;
        if (above + count([&](int i) { return key[i] == lo && place[i] <= mid; }) >= W) b = mid; else a = mid + 1;
    }
    return {lo, a};
}
template <class K>
__device__ __forceinline__ bool reaches(K key, uint32_t place, const Threshold<K>& t) { return key > t.key || (key == t.key && place <= t.place); }

// how many of the n candidates come before {key, place}
template <class K>
__device__ __forceinline__ int rank_of(const K* keys, const uint32_t* places, int n, K key, uint32_t place) {
    int r = 0;
    for (int i = 0; i < n; ++i) r += keys[i] > key || (keys[i] == key && places[i] < place);
    return r;
}

// whether beam w of prompt s has continuations to look for
__device__ __forceinline__ bool alive(const BeamParams& p, int64_t row) {
    return !(p.ended && p.ended[row]) && clean(p.scores[row]) != -INFINITY;
}

// A piece is NV times 16 bytes of every thread.  Pieces and threads go by the token, so that equal rows have equal sums wherever they
// begin: rows of an odd number of tokens are read from addresses that are multiples of an element's size only.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16, int NV>
__global__ void __launch_bounds__(kScanThreads)
beam_scan_kernel(BeamParams p) {
    constexpr int E = BF16 ? 2 : 4, PER = 16 / E, kWaves = kScanThreads / kWave, kMost = kMaxBeams * NV * PER;
    __shared__ float s_max[kWaves], s_sum[kWaves];
    __shared__ uint32_t s_key[kScanThreads], s_at[kScanThreads];
    __shared__ uint32_t s_ck[kMost], s_ca[kMost];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave;
    const DivMod rp = uniform_div_mod((int)blockIdx.x, p.by_pieces);
    const int64_t row = rp.q;
    if (!alive(p, row)) return;
    if (tid == 0) s_count = 0;

    const unsigned char* base = (const unsigned char*)p.logits + row * p.stride * E;
    const int first = rp.r * (kScanThreads * NV * PER) + tid * PER;      // token of the thread's first element
    float x[NV * PER];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int t0 = first + k * kScanThreads * PER;
        const unsigned char* at = base + (int64_t)t0 * E;
        uint32_t w[4] = {0, 0, 0, 0};
        if (t0 + PER <= p.V) {
            const u32x4_t y = *(const u32x4_t*)at;
            w[0] = y[0]; w[1] = y[1]; w[2] = y[2]; w[3] = y[3];
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const bool in = t0 + e < p.V;
                if constexpr (BF16) w[e / 2] |= (in ? (uint32_t)((const uint16_t*)at)[e] : 0xff80u) << (16 * (e % 2));
                else w[e] = in ? ((const uint32_t*)at)[e] : 0xff800000u;
            }
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (BF16) x[k * PER + e] = clean(__uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16));
            else x[k * PER + e] = clean(__uint_as_float(w[e]));
        }
    }
    // the thread's maximum and where it is first
    float top = x[0];
    int at = 0;
#pragma unroll
    for (int i = 1; i < NV * PER; ++i)
        if (x[i] > top) { top = x[i]; at = i; }
    s_key[tid] = key_of(top);
    auto token_of = [&](int i) { return (uint32_t)(first + i / PER * (kScanThreads * PER) + i % PER); };
    s_at[tid] = token_of(at);
    const float wm = wave_max(top);
    if (lane == 0) s_max[wv] = wm;
    __syncthreads();
    float m = s_max[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) m = fmaxf(m, s_max[i]);
    const float ref = m == -INFINITY ? 0.f : m;
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV * PER; ++i) part[i % 4] += __builtin_amdgcn_exp2f((x[i] - ref) * 1.4426950408889634f);
    float sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, kWave);
    if (lane == 0) s_sum[wv] = sum;

    const Threshold<uint32_t> t = nth_largest(s_key, s_at, kScanThreads, p.W, lane);
    if (reaches(s_key[tid], s_at[tid], t)) {
#pragma unroll
        for (int i = 0; i < NV * PER; ++i) {
            const uint32_t k = key_of(x[i]), a = token_of(i);
            if (k != 0 && reaches(k, a, t)) {
                const int c = atomicAdd(&s_count, 1);
                s_ck[c] = k;
                s_ca[c] = a;
            }
        }
    }
    __syncthreads();
    const int n = s_count;
    const int64_t list = (row * p.pieces + rp.r) * p.W;
    for (int i = tid; i < n; i += kScanThreads) {
        const uint32_t k = s_ck[i], a = s_ca[i];
        const int r = rank_of(s_ck, s_ca, n, k, a);
        if (r < p.W) {
            p.value[list + r] = __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
            p.token[list + r] = (int32_t)a;
        }
    }
    for (int i = n + tid; i < p.W; i += kScanThreads) p.token[list + i] = -1;
    if (tid == 0) {
        float all = s_sum[0];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) all += s_sum[i];
        p.sums[row * p.pieces + rp.r] = make_float2(m, all);
    }
}

__global__ void __launch_bounds__(kJoinThreads)
beam_join_kernel(BeamParams p) {
    constexpr int kWaves = kJoinThreads / kWave;
    __shared__ double s_off[kMaxBeams], s_score[kMaxBeams];
    __shared__ uint8_t s_ended[kMaxBeams];
    __shared__ uint64_t s_head[kMaxBeams * kMaxPieces], s_ck[kMaxBeams * kMaxBeams];
    __shared__ uint32_t s_place[kMaxBeams * kMaxPieces], s_ca[kMaxBeams * kMaxBeams];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid / kWave, W = p.W, n = W * p.pieces;
    const int64_t row0 = (int64_t)blockIdx.x * W;
    if (tid == 0) s_count = 0;
    for (int w = wv; w < W; w += kWaves) {
        const double score = (double)clean(p.scores[row0 + w]);
        const bool over = p.ended && p.ended[row0 + w], live = alive(p, row0 + w);
        double lse = 0.0;
        if (live) {
            float m = -INFINITY;
            for (int c = lane; c < p.pieces; c += kWave) m = fmaxf(m, p.sums[(row0 + w) * p.pieces + c].x);
            m = wave_max(m);
            double z = 0.0;
            for (int c = lane; c < p.pieces; c += kWave) {
                const float2 y = p.sums[(row0 + w) * p.pieces + c];
                if (y.x != -INFINITY) z += (double)y.y * exp((double)y.x - (double)m);
            }
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) z += __shfl_xor(z, d, kWave);
            lse = (double)m + log(z);
        }
        if (lane == 0) {
            s_off[w] = lse;
            s_score[w] = score;
            s_ended[w] = over ? 1 : live ? 0 : 2;                        // 2: no candidates
        }
    }
    __syncthreads();
    auto key = [&](int w, float x) { return key_of(((double)x - s_off[w]) + s_score[w]); };
    const uint32_t end = (uint32_t)max(p.end_token, 0);
    for (int i = tid; i < n; i += kJoinThreads) {
        const int w = i / p.pieces, c = i - w * p.pieces;
        uint64_t k = 0;
        uint32_t a = 0;
        if (s_ended[w] == 0) {
            const int64_t list = ((row0 + w) * p.pieces + c) * W;
            const int32_t t = p.token[list];
            if (t >= 0) { k = key(w, p.value[list]); a = (uint32_t)w * (uint32_t)p.V + (uint32_t)t; }
        } else if (s_ended[w] == 1 && c == 0) {
            k = key_of(s_score[w]);
            a = (uint32_t)w * (uint32_t)p.V + end;
        }
        s_head[i] = k;
        s_place[i] = a;
    }
    __syncthreads();
    const Threshold<uint64_t> t = nth_largest(s_head, s_place, n, W, lane);
    // (at most W lists have a first entry that reaches it, of W entries each)
    for (int i = tid; i < n * W; i += kJoinThreads) {
        const int l = i / W, e = i - l * W;
        if (s_head[l] == 0 || !reaches(s_head[l], s_place[l], t)) continue;
        const int w = l / p.pieces;
        uint64_t k = s_head[l];
        uint32_t a = s_place[l];
        if (e > 0) {
            if (s_ended[w] != 0) continue;
            const int64_t at = ((row0 + w) * p.pieces + (l - w * p.pieces)) * W + e;
            const int32_t tk = p.token[at];
            if (tk < 0) continue;
            k = key(w, p.value[at]);
            a = (uint32_t)w * (uint32_t)p.V + (uint32_t)tk;
            if (k == 0 || !reaches(k, a, t)) continue;
        }
        const int c = atomicAdd(&s_count, 1);
        s_ck[c] = k;
        s_ca[c] = a;
    }
    __syncthreads();
    const int found = s_count;
    for (int i = tid; i < found; i += kJoinThreads) {
        const uint64_t k = s_ck[i];
        const uint32_t a = s_ca[i];
        const int r = rank_of(s_ck, s_ca, found, k, a);
        if (r >= W) continue;
        const int w = (int)(a / (uint32_t)p.V), v = (int)(a - (uint32_t)w * (uint32_t)p.V);
        const bool over = s_ended[w] == 1;
        p.tokens[row0 + r] = over ? p.end_token : v;
        p.parents[row0 + r] = w;
        const uint64_t u = (k >> 63) ? k ^ (1ull << 63) : ~k;
        p.scores_out[row0 + r] = (float)__longlong_as_double((long long)u);
        if (p.ended_out) p.ended_out[row0 + r] = over || v == p.end_token;
    }
    for (int i = found + tid; i < W; i += kJoinThreads) {                // fewer continuations than beams
        p.tokens[row0 + i] = p.parents[row0 + i] = -1;
        p.scores_out[row0 + i] = -INFINITY;
        if (p.ended_out) p.ended_out[row0 + i] = 0;
    }
}

// Bytes of a piece over 4096
static int piece_vectors(int rows, int V, int esize) {
    for (int nv : {16, 8, 4})
        if ((int64_t)rows * V * esize >= (int64_t)nv * 4096 * 4 * compute_units()) return nv;
    return 2;
}
static int piece_count(int V, int esize, int nv) { return (int)(((int64_t)V * esize + nv * 4096 - 1) / (nv * 4096)); }
struct Pieces { int nv, count; };
static Pieces pieces_of(int rows, int V, int esize) {
    int nv = piece_vectors(rows, V, esize);
    while (piece_count(V, esize, nv) > kMaxPieces) nv *= 2;             // (16 always serves: kMaxV)
    return {nv, piece_count(V, esize, nv)};
}

bool beam_fits(int S, int W, int V, int esize) { return (int64_t)S * W * pieces_of(S * W, V, esize).count < 1 << 24; }

size_t beam_ws_bytes(int S, int W, int V, int esize) {
    const int64_t lists = (int64_t)S * W * pieces_of(S * W, V, esize).count;
    return (size_t)lists * (sizeof(float2) + (size_t)W * 8);
}

hipError_t launch_beam(int S, int W, int V, bool bf16, const void* logits, int64_t stride, const float* scores, const uint8_t* ended,
                       int end_token, int32_t* tokens, int32_t* parents, float* scores_out, uint8_t* ended_out, void* ws,
                       hipStream_t st) {
    const Pieces pc = pieces_of(S * W, V, bf16 ? 2 : 4);
    BeamParams p;
    p.S = S; p.W = W; p.V = V; p.pieces = pc.count; p.stride = stride;
    p.logits = logits; p.scores = scores; p.ended = ended; p.end_token = end_token;
    p.by_pieces = fast_div(pc.count);
    p.tokens = tokens; p.parents = parents; p.scores_out = scores_out; p.ended_out = ended_out;
    const int64_t lists = (int64_t)S * W * pc.count;
    p.sums = (float2*)ws;
    p.value = (float*)(p.sums + lists);
    p.token = (int32_t*)(p.value + lists * W);
    const dim3 grid((unsigned)lists), block(kScanThreads);
#define SCAN(NV) (bf16 ? beam_scan_kernel<true, NV> : beam_scan_kernel<false, NV>)
    auto* scan = pc.nv == 2 ? SCAN(2) : pc.nv == 4 ? SCAN(4) : pc.nv == 8 ? SCAN(8) : SCAN(16);
#undef SCAN
    hipLaunchKernelGGL(scan, grid, block, 0, st, p);
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)S), dim3(kJoinThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace pkv
