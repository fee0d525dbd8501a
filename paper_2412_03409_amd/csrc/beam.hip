// The W best continuations of a prompt's W beams: of beam w by token v
//   score(w, v) = scores[w] + x[w,v] - log sum_u exp x[w,u],
// equal ones by ascending w * V + v.  Within a beam the order is that of the logits, so a row's sum and its W largest logits come out
// of one pass, before its log-sum-exp is known; beams meet in a second, small launch.
//
//  beam_scan_kernel   a workgroup has a piece of a row, in registers: its maximum, the sum of its exponentials and its W largest logits.
//                     Which these are: W logits at least reach the W-th largest of the threads' maxima (or one up to W / 2 places
//                     below it, which is found in fewer steps), so only the threads whose maximum reaches it hold candidates, little more
//                     than W on the whole; each finds its rank by counting.
//                     Bound: HBM, one read of the logits; with 32 beams the choice beside it (about 590 vector instructions of a wavefront
//                     for 64 elements a lane).
//                     64 x 4 rows of 128000 in fp32 22.7 us (5.8 TB/s); 8 x 32 rows of 100003 in bf16 19.0 (2.7 TB/s); 4 rows of 32000 5.9.
//  beam_join_kernel   a workgroup has a prompt: maxima and sums of the rows from their pieces, then the same choice among the pieces'
//                     lists by their first entries.  Bound: dependent steps of one workgroup.  The same calls: 5.9, 10.3, 4.9 us.
//
// A sum of exponentials of a piece is held in 32 bits (terms of a thread, then a tree); pieces, logarithms and scores in 64, because
// beams are told apart by differences that 32 bits of a score of -10^2 do not hold.
#include "packed.hpp"
#include "fast_div.hpp"

namespace pkv {

constexpr int kScanThreads = 256;
constexpr int kWaveCandidates = 128;    // of a wavefront's part of a piece
constexpr int kManyFound = 512;         // candidates of a prompt beyond which those that cannot be are sorted out (4 prompts of 32 beams, 2729 tokens: 68 -> 20 us; 200 candidates: 24.5, 28.1 so)

struct BeamParams {
    int W, V, pieces;               // pieces of a row
    int group;                      // pieces, rounded up to a power of two
    int64_t stride;                 // of a row, in elements
    const void* logits;
    const float* scores;
    const uint8_t* ended;
    int end_token;                  // -1: none
    FastDiv by_pieces, by_w;
    int32_t *tokens, *parents;
    float* scores_out;
    uint8_t* ended_out;
    float2* sums;                   // workspace [S*W][pieces]: {maximum, sum of 2^(kLog2e x - base(maximum))}
    float* value;                   // workspace [S*W][pieces][W], descending
    int32_t* token;                 // the same, -1 behind the last
};

// NaN counts as -inf, +inf as the largest finite number
constexpr float kLargest = 3.402823466e38f;
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, kLargest); }
// an order-preserving whole number above 0 of a finite value, the same for both zeros; 0 stands for -inf: no candidate
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return x == -INFINITY ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// (of a key that no finite value has: the lowest one)
__device__ __forceinline__ float of_key(uint32_t k) {
    k = max(k, ~__float_as_uint(-kLargest));
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t key_of(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return x == -(double)INFINITY ? 0ull : (u >> 63) ? ~u : u | (1ull << 63);
}

// Terms of a row's sum are 2^(kLog2e x - base), one fma and one rounding of the exponent each; base = kLog2e * maximum, rounded, whose
// residue (exact in 32 bits) is taken off behind the sum.  Beyond kWideLogit the difference from the maximum is scaled: the residue, up to
// 2^-24 of the base, is an exponent of every term, which past 10^9 leaves the range and up to here stays below 2^-7.  (kLog2e is log2(e)
// but for 1.4e-8 of it: a sum's logarithm is off by that times the terms' mean distance from the maximum, which is log V at most: below 2e-7.)
// Nothing is added to a maximum: at 10^17 and beyond 64 bits would not hold the sum's logarithm next to it.
constexpr float kLog2e = 1.44269502f, kWideLogit = 65536.f;
constexpr double kLn2 = 0.693147180559945309417;
__device__ __forceinline__ float base_of(float m) { return m * kLog2e; }
// log of how much larger a sum is than that of exp(x - m)
__device__ __forceinline__ double residue_log(float m) { return fabsf(m) > kWideLogit ? 0.0 : (double)fmaf(m, kLog2e, -base_of(m)) * kLn2; }

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

// A threshold that the W largest of `n` entries {key, place} reach, and at most `slack` others: larger keys first, equal ones by ascending
// place, key 0: none.  Bisection over the keys that there are, by counting with ballots.  Every wavefront does it for itself, on entries
// in LDS or, the first 256, in registers.
template <class K>
struct Threshold { K key; uint32_t place; };
template <class K>
__device__ __forceinline__ bool reaches(K key, uint32_t place, const Threshold<K>& t) { return key > t.key || (key == t.key && place <= t.place); }

template <class K, class C>
__device__ __forceinline__ K nth_key(K lo, K hi, int W, int slack, C count) {       // count(k): entries of at least k; at least W reach lo
    while (lo < hi) {
        const K mid = lo + (hi - lo + 1) / 2;
        const int c = count(mid);
        if (c >= W && c <= W + slack) return mid;
        if (c > W) lo = mid; else hi = mid - 1;
    }
    return lo;
}
// in registers: R of a lane
template <int R, class K>
__device__ __forceinline__ K nth_key(const K (&k)[R], int W, int slack) {
    K lo = ~(K)0, hi = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) { hi = max(hi, k[i]); lo = min(lo, k[i] - 1); }        // (0 - 1 is the largest)
    hi = wave_max(hi);
    lo = wave_min(lo) + 1;
    auto count = [&](K x) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) c += __popcll(__builtin_amdgcn_ballot_w64(k[i] >= x));
        return c;
    };
    return hi == 0 || count(1) <= W ? (K)1 : nth_key(lo, hi, W, slack, count);
}
template <class K>
__device__ __forceinline__ Threshold<K> nth_largest(const K* key, const uint32_t* place, int n, int W, int slack, int lane) {
    auto count = [&](auto f) {
        int c = 0;
        for (int i = 0; i < n; i += kWave) c += __popcll(__builtin_amdgcn_ballot_w64(i + lane < n && f(min(i + lane, n - 1))));
        return c;
    };
    K t;
    if (n <= 4 * kWave) {
        K k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = i * kWave + lane < n ? key[i * kWave + lane] : 0;
        if constexpr (sizeof(K) == 8) {
            // the upper halves will mostly do
            uint32_t u[4];
            int c = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = (uint32_t)(k[i] >> 32);
            const uint32_t h = nth_key(u, W, slack);
#pragma unroll
            for (int i = 0; i < 4; ++i) c += __popcll(__builtin_amdgcn_ballot_w64(u[i] >= h));
            if (c <= W + slack) return {(K)h << 32, ~0u};
        }
        t = nth_key(k, W, slack);
    } else {
        K lo = ~(K)0, hi = 0;
        for (int i = lane; i < n; i += kWave) { hi = max(hi, key[i]); lo = min(lo, key[i] - 1); }
        hi = wave_max(hi);
        lo = wave_min(lo) + 1;
        auto at_least = [&](K x) { return count([&](int i) { return key[i] >= x; }); };
        t = hi == 0 || at_least(1) <= W ? (K)1 : nth_key(lo, hi, W, slack, at_least);
    }
    if (count([&](int i) { return key[i] >= t; }) <= W + slack) return {t, ~0u};
    const int above = count([&](int i) { return key[i] > t; });
    uint32_t a = 0, b = ~0u;                                             // the lowest places of the equal ones
    while (a < b) {
        const uint32_t mid = a + (b - a) / 2;
        if (above + count([&](int i) { return key[i] == t && place[i] <= mid; }) >= W) b = mid; else a = mid + 1;
    }
    return {t, a};
}

__device__ __forceinline__ uint32_t of_lane(uint32_t x, int j) { return (uint32_t)__builtin_amdgcn_readlane((int)x, j); }
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int j) { return ((uint64_t)of_lane((uint32_t)(x >> 32), j) << 32) | of_lane((uint32_t)x, j); }
// how many of the n candidates come before this lane's, where a wavefront holds them all
template <class K>
__device__ __forceinline__ int rank_in_wave(int n, K key, uint32_t place) {
    int r = 0;
    for (int j = 0; j < n; ++j) {
        const K k = of_lane(key, j);
        const uint32_t a = of_lane(place, j);
        r += (k > key) | ((k == key) & (a < place));
    }
    return r;
}
// A piece is NV times 16 bytes of every thread.  Pieces and threads go by the token, so that equal rows have equal sums wherever they
// begin: rows of an odd number of tokens are read from addresses that are multiples of an element's size only.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4), aligned(2)));
template <bool BF16, int NV>
__global__ void __launch_bounds__(kScanThreads, 4)
beam_scan_kernel(BeamParams p) {
    constexpr int E = BF16 ? 2 : 4, PER = 16 / E, N = NV * PER, kWaves = kScanThreads / kWave, kPiece = kScanThreads * N;
    constexpr int kMost = kMaxBeams * N > kWaves * kWaveCandidates ? kMaxBeams * N : kWaves * kWaveCandidates;
    __shared__ float s_sum[kWaves];
    __shared__ uint32_t s_key[kScanThreads], s_at[kScanThreads];
    // candidates (two arrays: a store of both together would want every element in a pair of registers)
    __shared__ float s_v[kMost];
    __shared__ int s_t[kMost];
    __shared__ int s_n[kWaves], s_count;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(tid / kWave);
    const DivMod rp = uniform_div_mod((int)blockIdx.x, p.by_pieces);
    const int64_t row = rp.q;
    const unsigned char* base = (const unsigned char*)p.logits + row * p.stride * E;
    const int first = rp.r * kPiece + tid * PER;                         // token of the thread's first element
    auto token_of = [&](int i) { return first + i / PER * (kScanThreads * PER) + i % PER; };
    auto load = [&](int t) {
        if constexpr (BF16) return __uint_as_float((uint32_t)((const uint16_t*)base)[t] << 16);
        else return ((const float*)base)[t];
    };
    // Where a launch is small its latency counts, and the logits are asked for ahead of whether they are needed.
    const uint8_t over = p.ended ? p.ended[row] : 0;
    const float score = p.scores[row];
    auto dead = [&]() { return over != 0 || clean(score) == -INFINITY; };
    if (NV > 2 && dead()) return;
    float x[N];
    auto unpack = [&](int k, const u32x4_t& y) {
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if constexpr (BF16) x[k * PER + e] = __uint_as_float(e % 2 ? y[e / 2] & 0xffff0000u : y[e / 2] << 16);
            else x[k * PER + e] = __uint_as_float(y[e]);
        }
    };
    if (rp.r * kPiece + kPiece <= p.V) {                                 // a whole piece
#pragma unroll
        for (int k = 0; k < NV; ++k) unpack(k, *(const u32x4_t*)(base + (int64_t)token_of(k * PER) * E));
    } else {
        // threads begin at multiples of PER: one of them has the row's last elements
        const int end = p.V - p.V % PER;
        const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;
        u32x4_t last = {none, none, none, none};
#pragma unroll
        for (int e = 0; e + 1 < PER; ++e)
            if (end + e < p.V) {
                if constexpr (BF16) last[e / 2] = (last[e / 2] & (0xffffu << (16 * (1 - e % 2)))) | (uint32_t)((const uint16_t*)base)[end + e] << (16 * (e % 2));
                else last[e] = ((const uint32_t*)base)[end + e];
            }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int t0 = token_of(k * PER);
            u32x4_t y = {none, none, none, none};
            if (t0 < end) y = *(const u32x4_t*)(base + (int64_t)t0 * E);
            else if (t0 == end) y = last;
            unpack(k, y);
        }
    }
    if (NV <= 2 && dead()) return;
    // The largest, or NaN if there is one: one look tells whether the wavefront has any value that counts as another.
    auto largest = [&]() {
        float v = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) v = __builtin_elementwise_maximum(v, x[i]);
        return v;
    };
    float top = largest();
    if (__builtin_amdgcn_ballot_w64(!(top <= kLargest)) != 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = clean(x[i]);
        top = largest();
    }
    s_key[tid] = key_of(top);
    __syncthreads();
    uint32_t keys[kWaves], most = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        keys[i] = s_key[i * kWave + lane];
        most = max(most, keys[i]);
    }
    most = wave_max(most);
    const float m = most == 0 ? -INFINITY : of_key(most);

    float part[4] = {0.f, 0.f, 0.f, 0.f};
    if (fabsf(m) > kWideLogit) {
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < N; ++i) part[i % 4] += __builtin_amdgcn_exp2f((x[i] - ref) * kLog2e);
    } else {
        const float ref = base_of(m);
#pragma unroll
        for (int i = 0; i < N; ++i) part[i % 4] += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, -ref));
    }
    float sum = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, kWave);

    // Candidates are what reaches the W-th largest of the threads' maxima: few more than W.
    const uint32_t t = nth_key(keys, p.W, p.W / 2);
    const float least = of_key(t);
    int got = 0;                                                         // of the wavefront
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool is = x[i] >= least;
        const unsigned long long who = __builtin_amdgcn_ballot_w64(is);
        if (who != 0) {
            const int at = got + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
            if (is && at < kWaveCandidates) {
                s_v[wv * kWaveCandidates + at] = x[i];
                s_t[wv * kWaveCandidates + at] = token_of(i);
            }
            got += (int)__popcll(who);
        }
    }
    if (lane == 0) { s_sum[wv] = sum; s_n[wv] = got; }
    __syncthreads();
    const int64_t list = (row * p.pieces + rp.r) * p.W;
    int n[kWaves], all = 0;
    bool many = false;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) { n[i] = s_n[i]; all += n[i]; many = many || n[i] > kWaveCandidates; }
    auto give = [&](float v, int tk, int r) {
        if (r < p.W) {
            p.value[list + r] = v;
            p.token[list + r] = tk;
        }
    };
    auto before = [&](float v, int tk, int from, int count) {            // candidates that come before
        int r = 0;
#pragma unroll 4
        for (int j = from; j < from + count; ++j) r += (s_v[j] > v) | ((s_v[j] == v) & (s_t[j] < tk));
        return r;
    };
    if (!many && all <= kWave) {
        // one wavefront has them all
        if (wv != 0) return;
        float v = 0.f;
        int tk = 0, at = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (lane >= at && lane < at + n[w]) {
                v = s_v[w * kWaveCandidates + lane - at];
                tk = s_t[w * kWaveCandidates + lane - at];
            }
            at += n[w];
        }
        const int r = rank_in_wave(all, key_of(v), (uint32_t)tk);
        if (lane < all) give(v, tk, r);
    } else if (!many) {
        // a quarter of the candidates at a time: rank by counting
        for (int i = lane; i < n[wv]; i += kWave) {
            const float v = s_v[wv * kWaveCandidates + i];
            const int tk = s_t[wv * kWaveCandidates + i];
            int r = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) r += before(v, tk, w * kWaveCandidates, n[w]);
            give(v, tk, r);
        }
    } else {
        // Many equal logits: of those the lowest tokens, W threads' at most, whose elements are read again.
        int at = 0;
#pragma unroll
        for (int i = N - 1; i >= 0; --i) at = x[i] == top ? i : at;
        s_at[tid] = (uint32_t)token_of(at);
        if (tid == 0) s_count = 0;
        __syncthreads();
        const Threshold<uint32_t> te = nth_largest(s_key, s_at, kScanThreads, p.W, 0, lane);
        if (reaches(s_key[tid], s_at[tid], te)) {
#pragma unroll 4
            for (int i = 0; i < N; ++i) {
                const int tk = token_of(i);
                const float v = tk < p.V ? clean(load(tk)) : -INFINITY;
                if (v != -INFINITY && reaches(key_of(v), (uint32_t)tk, te)) {
                    const int at = atomicAdd(&s_count, 1);
                    s_v[at] = v;
                    s_t[at] = tk;
                }
            }
        }
        __syncthreads();
        all = s_count;
        for (int i = tid; i < all; i += kScanThreads) give(s_v[i], s_t[i], before(s_v[i], s_t[i], 0, all));
    }
    for (int i = all + tid; i < p.W; i += kScanThreads) p.token[list + i] = -1;
    if (tid == 0) p.sums[row * p.pieces + rp.r] = make_float2(m, (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
}

// Which of the candidates of a workgroup, R of a thread, are among the W best, and at most 64 - W others: bisection over the upper halves
// of the scores, where equal ones are too many over the lower halves, and then over the places.  Every step is a count of the whole workgroup.
template <int THREADS, int R>
struct Best {
    int* counts;                        // LDS, 0
    int lane, step, W;
    // v: larger ones first; in: whether it takes part; above: how many come before those.  -> which take part, at least W - above of them
    __device__ __forceinline__ bool narrow(const uint32_t (&v)[R], bool (&in)[R], int& above) {
        uint32_t lo = 0, hi = ~0u;
        int at_lo = -1;                                                  // how many reach lo
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            int c = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) c += __popcll(__builtin_amdgcn_ballot_w64(in[r] && v[r] >= mid));
            c = above + all(c);
            if (c >= W) { lo = mid; at_lo = c; } else hi = mid - 1;
            if (c >= W && c <= kWave) break;
        }
        const bool enough = at_lo >= 0 && at_lo <= kWave;
        int more = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            more += enough ? 0 : __popcll(__builtin_amdgcn_ballot_w64(in[r] && v[r] > lo));
            sure[r] = sure[r] || (in[r] && (enough ? v[r] >= lo : v[r] > lo));
            in[r] = !enough && in[r] && v[r] == lo;
        }
        if (!enough) above += all(more);
        return enough;
    }
    __device__ __forceinline__ int all(int c) {                          // sum over the workgroup's wavefronts
        if (lane == 0) atomicAdd(counts + step, c);
        __syncthreads();
        return counts[step++];
    }
    bool sure[R];                       // the verdict
};

// A group of lanes, a power of two of them, has the pieces of a row.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
beam_join_kernel(BeamParams p) {
    constexpr int kHeads = (kMaxBeams * kMaxPieces + 1023) / 1024;       // of a thread, at most
    constexpr int kLists = kMaxBeams * 3 / 2, R = 2, kSteps = 3 * 34;
    static_assert(1024 * R >= kLists * kMaxBeams, "a thread has R of what the lists hold");
    __shared__ double s_log[kMaxBeams], s_score[kMaxBeams];             // log of the sum of exp(x - maximum)
    __shared__ float s_max[kMaxBeams];
    __shared__ uint8_t s_kind[kMaxBeams];                                // 0: goes on, 1: has ended, 2: no candidates
    __shared__ uint64_t s_head[kMaxBeams * kMaxPieces], s_ck[kLists * kMaxBeams];
    __shared__ uint32_t s_place[kMaxBeams * kMaxPieces], s_ca[kLists * kMaxBeams];
    __shared__ Threshold<uint64_t> s_t;
    __shared__ int s_list[kLists], s_lists, s_count, s_counts[kSteps];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), W = p.W, n = W * p.pieces;
    const bool first_wave = tid < kWave;
    const int64_t row0 = (int64_t)blockIdx.x * W;
    if (tid == 0) s_count = 0;
    // the lists' first entries are asked for ahead of the sums (those of rows that are not looked at hold anything)
    float hv[kHeads];
    int32_t ht[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int64_t at = (row0 * p.pieces + min(tid + i * THREADS, n - 1)) * W;
        hv[i] = p.value[at];
        ht[i] = p.token[at];
    }
    const int c = tid & (p.group - 1);
    for (int w = tid / p.group; w < W; w += THREADS / p.group) {         // (a wavefront's lanes leave the loop together or by groups)
        const double score = (double)clean(p.scores[row0 + w]);
        const bool over = p.ended && p.ended[row0 + w], live = !over && score != -(double)INFINITY;
        float2 y = make_float2(-INFINITY, 0.f);
        if (live && c < p.pieces) y = p.sums[(row0 + w) * p.pieces + c];
        float m = y.x;                                                   // (a row without candidates: its sum is not used)
        for (int d = p.group / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, kWave));
        double z = y.x != -INFINITY ? (double)y.y * exp(((double)y.x - (double)m) - residue_log(y.x)) : 0.0;
        for (int d = p.group / 2; d > 0; d >>= 1) z += __shfl_xor(z, d, kWave);
        if (c == 0) {
            s_max[w] = m;
            s_log[w] = live ? log(z) : 0.0;
            s_score[w] = score;
            s_kind[w] = over ? 1 : live ? 0 : 2;
        }
    }
    __syncthreads();
    auto key = [&](int w, float x) { return key_of((((double)x - (double)s_max[w]) - s_log[w]) + s_score[w]); };
    auto place = [&](int w, int v) { return (uint32_t)w * (uint32_t)p.V + (uint32_t)v; };
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        const int l = tid + i * THREADS;
        if (l >= n) break;
        const DivMod wc = div_mod(l, p.by_pieces);
        const int w = wc.q;
        uint64_t k = 0;
        uint32_t a = 0;
        if (s_kind[w] == 0 && ht[i] >= 0) {
            k = key(w, hv[i]);
            a = place(w, ht[i]);
        } else if (s_kind[w] == 1 && wc.r == 0) {
            k = key_of(s_score[w]);
            a = place(w, max(p.end_token, 0));
        }
        s_head[l] = k;
        s_place[l] = a;
    }
    __syncthreads();
    if (first_wave) {
        const Threshold<uint64_t> t = nth_largest(s_head, s_place, n, W, W / 2, lane);
        int got = 0;                                                     // W + W/2 lists at most
        for (int i = 0; i < n; i += kWave) {
            const int l = min(i + lane, n - 1);
            const bool is = i + lane < n && s_head[l] != 0 && reaches(s_head[l], s_place[l], t);
            const unsigned long long who = __builtin_amdgcn_ballot_w64(is);
            if (is) s_list[got + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = l;
            got += (int)__popcll(who);
        }
        if (lane == 0) { s_t = t; s_lists = got; }
    }
    __syncthreads();
    const Threshold<uint64_t> t = s_t;
    const int all = s_lists * W;
    for (int i = tid; i < all; i += THREADS) {
        const DivMod le = div_mod(i, p.by_w);
        const int l = s_list[le.q], w = div_mod(l, p.by_pieces).q;
        uint64_t k = s_head[l];
        uint32_t a = s_place[l];
        if (le.r > 0) {
            if (s_kind[w] != 0) continue;
            const int64_t at = (row0 * p.pieces + l) * W + le.r;
            const int32_t v = p.token[at];
            const float x = p.value[at];
            if (v < 0) continue;
            k = key(w, x);
            a = place(w, v);
            if (k == 0 || !reaches(k, a, t)) continue;
        }
        const int at = atomicAdd(&s_count, 1);
        s_ck[at] = k;
        s_ca[at] = a;
    }
    __syncthreads();
    int found = s_count;
    auto give = [&](uint64_t k, uint32_t a, int r) {
        if (r >= W) return;
        const int w = (int)(a / (uint32_t)p.V), v = (int)(a - (uint32_t)w * (uint32_t)p.V);
        const bool over = s_kind[w] == 1;
        p.tokens[row0 + r] = over ? p.end_token : v;
        p.parents[row0 + r] = w;
        const uint64_t u = (k >> 63) ? k ^ (1ull << 63) : ~k;
        p.scores_out[row0 + r] = (float)__longlong_as_double((long long)u);
        if (p.ended_out) p.ended_out[row0 + r] = over || v == p.end_token;
    };
    if (THREADS == 1024 && found > kManyFound) {
        // a few beams have most of them: what is not among the W best leaves
        uint64_t k[R];
        uint32_t a[R], part[R];
        Best<THREADS, R> best{s_counts, lane, 0, W, {}};
        bool in[R];
        int above = 0;
        for (int i = tid; i < kSteps; i += THREADS) s_counts[i] = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = tid + r * THREADS;
            in[r] = i < found;
            best.sure[r] = false;
            k[r] = in[r] ? s_ck[i] : 0;
            a[r] = in[r] ? s_ca[i] : 0;
            part[r] = (uint32_t)(k[r] >> 32);
        }
        __syncthreads();
        if (!best.narrow(part, in, above)) {
#pragma unroll
            for (int r = 0; r < R; ++r) part[r] = (uint32_t)k[r];
            if (!best.narrow(part, in, above)) {
#pragma unroll
                for (int r = 0; r < R; ++r) part[r] = ~a[r];
                best.narrow(part, in, above);
            }
        }
        if (tid == 0) s_count = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (best.sure[r]) {
                const int at = atomicAdd(&s_count, 1);
                s_ck[at] = k[r];
                s_ca[at] = a[r];
            }
        __syncthreads();
        found = s_count;
    }
    if (found <= kWave) {
        if (!first_wave) return;
        const uint64_t k = lane < found ? s_ck[lane] : 0;
        const uint32_t a = lane < found ? s_ca[lane] : 0;
        const int r = rank_in_wave(found, k, a);
        if (lane < found) give(k, a, r);
    } else {
        // as many lanes as there are have a candidate, up to eight
        int g = 8;
        while (g > 1 && found * g > THREADS) g /= 2;
        for (int i0 = 0; i0 < found; i0 += THREADS / g) {
            const int i = i0 + tid / g;
            const uint64_t k = s_ck[min(i, found - 1)];
            const uint32_t a = s_ca[min(i, found - 1)];
            int r = 0;
#pragma unroll 4
            for (int j = tid & (g - 1); j < found; j += g) r += (s_ck[j] > k) | ((s_ck[j] == k) & (s_ca[j] < a));
            for (int d = 1; d < g; d <<= 1) r += __shfl_xor(r, d, kWave);
            if ((tid & (g - 1)) == 0 && i < found) give(k, a, r);
        }
    }
    for (int i = found + tid; i < W; i += THREADS) {                     // fewer continuations than beams (and than lanes)
        p.tokens[row0 + i] = p.parents[row0 + i] = -1;
        p.scores_out[row0 + i] = -INFINITY;
        if (p.ended_out) p.ended_out[row0 + i] = 0;
    }
}

// A piece is nv * 4096 bytes: 64 elements of a thread at most, which are registers, fewer where the launch would have less than a
// workgroup for each compute unit.  (16 x 4 rows of 128000 in bf16: 12.6 us so, 15.6 with four of them; 64 elements, not 32: 256 rows of
// 100003 29.1 us, 33.8.)
struct Pieces { int nv, count; };
static Pieces pieces_of(int rows, int V, int esize) {
    const int most = esize == 4 ? 16 : 8;
    int nv = most;
    while (nv > 2 && (int64_t)rows * V * esize < (int64_t)nv * 4096 * compute_units()) nv /= 2;
    auto count = [&]() { return (int)(((int64_t)V * esize + nv * 4096 - 1) / (nv * 4096)); };
    while (count() > kMaxPieces) nv *= 2;                               // (not beyond `most`: kMaxV)
    // as few as that number of pieces needs (in fp32 an even number): all elements take part in the choice, also those that are not there.
    // (us, at most / as few: 352 rows of 26754 in fp32 29.8 / 25.9, 232 of 35111 17.4 / 15.3, 256 of 100003 in bf16 29.6 / 27.8)
    const int pieces = count(), step = esize == 4 ? 2 : 1;
    while (nv > 2 && (nv -= step, count() == pieces)) {}
    if (count() != pieces) nv += step;
    return {nv, pieces};
}

// workgroups are counted in 24 bits, as a grid's threads (256 of a workgroup) are in 32
static_assert((int64_t)kMaxS * kMaxBeams * kMaxPieces < 1 << 24, "any call's pieces are a grid");

size_t beam_ws_bytes(int S, int W, int V, int esize) {
    const int64_t lists = (int64_t)S * W * pieces_of(S * W, V, esize).count;
    return (size_t)lists * (sizeof(float2) + (size_t)W * 8);
}

hipError_t launch_beam(int S, int W, int V, bool bf16, const void* logits, int64_t stride, const float* scores, const uint8_t* ended,
                       int end_token, int32_t* tokens, int32_t* parents, float* scores_out, uint8_t* ended_out, void* ws,
                       hipStream_t st) {
    const Pieces pc = pieces_of(S * W, V, bf16 ? 2 : 4);
    BeamParams p;
    p.W = W; p.V = V; p.pieces = pc.count; p.stride = stride;
    p.logits = logits; p.scores = scores; p.ended = ended; p.end_token = end_token;
    p.by_pieces = fast_div(pc.count); p.by_w = fast_div(W);
    p.group = 1;
    while (p.group < pc.count) p.group *= 2;
    p.tokens = tokens; p.parents = parents; p.scores_out = scores_out; p.ended_out = ended_out;
    const int64_t lists = (int64_t)S * W * pc.count;
    p.sums = (float2*)ws;
    p.value = (float*)(p.sums + lists);
    p.token = (int32_t*)(p.value + lists * W);
    const dim3 grid((unsigned)lists), block(kScanThreads);
    static constexpr void (*kScan16[])(BeamParams) = {beam_scan_kernel<true, 2>, beam_scan_kernel<true, 3>, beam_scan_kernel<true, 4>, beam_scan_kernel<true, 5>,
                                                      beam_scan_kernel<true, 6>, beam_scan_kernel<true, 7>, beam_scan_kernel<true, 8>};
    static constexpr void (*kScan32[])(BeamParams) = {beam_scan_kernel<false, 2>, beam_scan_kernel<false, 4>, beam_scan_kernel<false, 6>, beam_scan_kernel<false, 8>,
                                                      beam_scan_kernel<false, 10>, beam_scan_kernel<false, 12>, beam_scan_kernel<false, 14>, beam_scan_kernel<false, 16>};
    auto* scan = bf16 ? kScan16[pc.nv - 2] : kScan32[pc.nv / 2 - 1];
    hipLaunchKernelGGL(scan, grid, block, 0, st, p);
    if (W <= 4) hipLaunchKernelGGL(beam_join_kernel<256>, dim3((unsigned)S), dim3(256), 0, st, p);
    else hipLaunchKernelGGL(beam_join_kernel<1024>, dim3((unsigned)S), dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace pkv
