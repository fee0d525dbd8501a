// Causal attention of packed rows: whole prompts of different lengths over their own packed keys, and chunks of new rows over a
// paged cache.  Both are one operator with two places to read keys from: row i of a sequence's n rows sees the keys
// 0 ... len - n + i, where len = n for a prompt.  Query heads that share a KV head are rows of one tile, row = token * heads + head:
// the keys are read once for all of them, and a tile's diagonal is as narrow as its tokens are few.
//
//  attn_tiles_kernel  bf16, many rows.  A workgroup has 128 rows of one (sequence, KV head), a wavefront 32 of them.  Keys and
//                     values stream through LDS 64 at a time (asynchronous copies, two buffer pairs).  Bound: the matrix cores
//                     and the softmax next to them; four prompts of 8192 rows, H32/8, D128: 2.1 to 2.2 ms, 1 PFLOP/s.  Short prompts:
//                     the longest tile, 1.27 us a stage and about 6 us to begin and end (680 rows of 32 heads 19 to 20 us).
//  attn_stream_kernel bf16, at most 32 rows per (sequence, KV head): decode steps.  A wavefront streams 32 keys at a time through
//                     LDS of its own.  All keys of a launch are one sequence of blocks that the wavefronts share out evenly,
//                     wherever the units begin and end.  Bound: HBM; 467 MB of keys and values of 32 sequences in 90 us, 5.2 TB/s
//                     (a plain read reaches 5.8), and 5 us to join.
//  attn_merge_*       join the parts of a tile or unit that several workgroups or wavefronts worked on.
//  attn_rows_kernel   fp32: a workgroup per (row, head, layer).  The keys stream past one row: LPR lanes hold a key
//                     row, scores meet by shuffles, softmax online (running maximum and sum, everything fp32); the four
//                     wavefronts take every fourth group of keys and join through LDS (one wavefront for all keys 11.5 us, so 6.6,
//                     15 rows over up to 136 keys, 4 layers).  Bound: latency at the sizes of the fp32 validation shape.
//
// The two bf16 kernels work as the prompt attention of rectangular batches does: S^T[32 keys x 32 rows] = K Q^T and
// O^T[32 columns x 32 rows] += V^T P^T with v_mfma_f32_32x32x16_bf16.  A lane holds one row's scores, so the softmax state is a
// scalar per lane, and the probabilities, as bf16 against the running maximum (the stream kernel: as two bf16 numbers each), are the
// second product's operand where they are.  V^T comes from row-major V by the transposing LDS read.
#include "packed.hpp"
#include "fast_div.hpp"
#include "packed_rules.hpp"

namespace pkv {

struct PackedParams {
    int S, L, H, Hkv, T;
    int grp;                        // H / Hkv
    int num_pages, max_pages, shift, layers, l0, max_rows;
    const unsigned char *q, *k, *v;
    unsigned char* out;
    Strides qs, ks, vs, os;         // in bytes
    const int32_t *row_off, *table, *lens;
    const float* scale;
    float* lse;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The logit scale's size; its sign goes into the queries (exact), so that maxima can be taken on the products.  Above 0, so that a masked
// -inf stays one: the smallest number there is, times the largest score, is still below 2^-20 (NaN stays NaN).
__device__ __forceinline__ float scale_size(float sc) {
    const float a = fabsf(sc);
    return a < 1.401298464e-45f ? 1.401298464e-45f : a;
}
// The same in units of log2: a weight is 2^((score - maximum) * this).  Scores are scaled behind their difference, because the largest
// finite ones leave the range when they are scaled, and lose whole units in the rounding: rows whose keys all score the type's lowest
// value weigh them equally.
__device__ __forceinline__ float score_scale(float sc) { return scale_size(sc) * kLog2e; }

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, kWave);
    return x;
}

// entries that segment (s, layer l of the call) holds
__device__ __forceinline__ int entries(const PackedParams& p, int s, int l) {
    const int len = p.lens[(int64_t)s * p.layers + p.l0 + l];
    return max(0, min(len, p.max_pages << p.shift));
}

// ---- fp32 ----------------------------------------------------------------------------------------------
template <int D>
__global__ void __launch_bounds__(256)
attn_rows_kernel(PackedParams p) {
    constexpr int LPR = D / 4, RG = kWave / LPR, U = 4, kRow = D * 4;
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave, sub = lane % LPR, rg = lane / LPR;
    const int t = blockIdx.x, h = blockIdx.y, l = blockIdx.z;
    // the sequence of row t: how many end at t or before it
    int s = 0;
    for (int i = lane; i < p.S; i += kWave) s += p.row_off[i + 1] <= t;
    s = wave_sum(s);
    if (s >= p.S) return;
    const int first = p.row_off[s], n = p.row_off[s + 1] - first, i = t - first;
    if (first < 0 || i < 0 || i >= p.max_rows) return;
    const int len = entries(p, s, l), count = min(len, i + 1 + len - n);    // keys that the row sees
    const int32_t* pages = p.table + ((int64_t)s * p.layers + p.l0 + l) * p.max_pages;
    const int g = h / p.grp;
    float4 q = *(const float4*)(p.q + p.qs.l * l + p.qs.h * h + p.qs.n * t + sub * 16);
    const float sc0 = p.scale[l], scale = score_scale(sc0);
    if (sc0 < 0.f) q = make_float4(-q.x, -q.y, -q.z, -q.w);
    float m = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto weigh = [](float4& x, float c) { x.x *= c; x.y *= c; x.z *= c; x.w *= c; };
    for (int j0 = wv * RG * U; j0 < count; j0 += 4 * RG * U) {
        float4 kr[U], vr[U];
        bool real[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * RG + rg;
            const int id = j < count ? pages[j >> p.shift] : -1;
            real[u] = (uint32_t)id < (uint32_t)p.num_pages;
            kr[u] = vr[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (real[u]) {
                const int64_t at = ((((int64_t)id * p.Hkv + g) << p.shift) + (j & ((1 << p.shift) - 1))) * kRow + sub * 16;
                kr[u] = *(const float4*)(p.k + at);
                vr[u] = *(const float4*)(p.v + at);
            }
        }
        float sc[U], mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float d = fmaf(q.x, kr[u].x, fmaf(q.y, kr[u].y, fmaf(q.z, kr[u].z, q.w * kr[u].w)));
#pragma unroll
            for (int x = 1; x < LPR; x <<= 1) d += __shfl_xor(d, x, kWave);
            sc[u] = real[u] ? d : -INFINITY;
            mx = fmaxf(mx, sc[u]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx, corr = __builtin_amdgcn_exp2f((m - ref) * scale);
        m = mx;
        sum *= corr;
        weigh(o, corr);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = __builtin_amdgcn_exp2f((sc[u] - ref) * scale);
            sum += w;
            o.x = fmaf(w, vr[u].x, o.x); o.y = fmaf(w, vr[u].y, o.y); o.z = fmaf(w, vr[u].z, o.z); o.w = fmaf(w, vr[u].w, o.w);
        }
    }
    // the row groups hold every RG-th key each
    float all = m;
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) all = fmaxf(all, __shfl_xor(all, x, kWave));
    const float ref = all == -INFINITY ? 0.f : all, corr = __builtin_amdgcn_exp2f((m - ref) * scale);
    sum *= corr;
    weigh(o, corr);
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) {
        sum += __shfl_xor(sum, x, kWave);
        o.x += __shfl_xor(o.x, x, kWave); o.y += __shfl_xor(o.y, x, kWave);
        o.z += __shfl_xor(o.z, x, kWave); o.w += __shfl_xor(o.w, x, kWave);
    }
    __shared__ float2 s_ms[4];
    __shared__ float4 s_o[4][LPR];
    if (lane == 0) s_ms[wv] = make_float2(all, sum);
    if (rg == 0) s_o[wv][sub] = o;
    __syncthreads();
    if (wv != 0 || rg != 0) return;
    float top = all;
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, s_ms[w].x);
    const float base = top == -INFINITY ? 0.f : top, mine = __builtin_amdgcn_exp2f((all - base) * scale);
    sum *= mine;
    weigh(o, mine);
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float2 ms = s_ms[w];
        const float4 y = s_o[w][sub];
        const float c = __builtin_amdgcn_exp2f((ms.x - base) * scale);
        sum = fmaf(ms.y, c, sum);
        o.x = fmaf(y.x, c, o.x); o.y = fmaf(y.y, c, o.y); o.z = fmaf(y.z, c, o.z); o.w = fmaf(y.w, c, o.w);
    }
    weigh(o, sum == 0.f ? 0.f : 1.f / sum);                     // nothing seen: zeros
    *(float4*)(p.out + p.os.l * l + p.os.h * h + p.os.n * t + sub * 16) = o;
}

// ---- bf16: the matrix cores ----------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef unsigned short v2u16_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4i16_t lds_v4i16_t;

constexpr int kTileRows = 128;      // rows of a workgroup
constexpr int kStage = 64;          // keys that a workgroup stages at a time
constexpr int kBlockKeys = 32;      // keys that a wavefront of the stream kernel takes at a time
constexpr int kFewRows = 32;        // rows of a unit of the stream kernel
constexpr float kWide = 4096.f;     // scaled scores beyond are scaled behind their difference

// 4 keys of one column of row-major V (lane i of a group of 16 receives column i of the 4 keys that the group points at)
__device__ __forceinline__ v4i16_t lds_read_tr(const unsigned char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)p);
}

// Chunk c of staged row r sits at c ^ swz(r): rows of 16 at one chunk (K) and 4 rows at 4 chunks (V) then meet no bank twice.
template <int CPR>
__device__ __forceinline__ int swz(int r) {
    if constexpr (CPR == 16) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return ((r & 1) << 2) | ((r >> 1) & 3);
}

// Where a lane copies from when 16 rows go to LDS, 1 KB at a time: lane i of copy x writes 16 bytes at 1024 x + 16 i, that is
// chunk i % CPR of row x * 64 / CPR + i / CPR, which holds the row's chunk that the swizzle moves there.
template <int D>
struct CopyLane {
    static constexpr int CPR = D / 8, RPC = kWave / CPR, kCopies = 16 / RPC;
    uint32_t row, col;                        // of copy 0; column in bytes
    __device__ __forceinline__ explicit CopyLane(int lane) {
        row = (uint32_t)(lane / CPR);
        col = 16u * (uint32_t)((lane % CPR) ^ swz<CPR>(lane / CPR));
        asm volatile("" : "+v"(row), "+v"(col));
    }
    // byte offset of copy x; rows from `last` on are read like row `last`
    __device__ __forceinline__ uint32_t at(int x, uint32_t last, uint32_t row_bytes) const {
        const uint32_t r = min(row + (uint32_t)(x * RPC), last);
        return r * row_bytes + (CPR == 16 ? col ^ (16u * (uint32_t)x) : col);      // (rows a multiple of 8 apart are swizzled alike if CPR is 8)
    }
};

__device__ __forceinline__ void copy_to_lds(const unsigned char* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// 32 columns of 32 finished rows: register r is column 8 (r / 4) + 4 (lane / 32) + r % 4.  16 bytes per lane and 8 columns: the
// halves of a row swap their pieces.
__device__ __forceinline__ void store_columns(const f32x16_t& o, unsigned char* row, int hf, float inv, bool real) {
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
        uint32_t w[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            w[x][0] = pack_bf16(o[4 * (g + x)] * inv, o[4 * (g + x) + 1] * inv);
            w[x][1] = pack_bf16(o[4 * (g + x) + 2] * inv, o[4 * (g + x) + 3] * inv);
        }
        const auto s0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
        const auto s1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
        if (real) *(uint4*)(row + 2 * (8 * (g + hf))) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
}

// Whether `count` KB of staged values, at 1 KB a read of the wavefront, hold one that is infinite or NaN.
template <int COUNT>
__device__ __forceinline__ bool wild_values(const unsigned char* sV, int lane) {
    v2u16_t big = {0, 0};
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const uint4 w = *(const uint4*)(sV + i * 1024 + lane * 16);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) big = __builtin_elementwise_max(big, __builtin_bit_cast(v2u16_t, x[e] & 0x7fff7fffu));
    }
    return __builtin_amdgcn_ballot_w64(big.x >= 0x7f80 || big.y >= 0x7f80) != 0;
}

// Softmax state and output of the 32 rows of a wavefront: row lane % 32; register r of o[dt] is column
// 32 dt + 8 (r / 4) + 4 (lane / 32) + r % 4.
template <int D>
struct RowTile {
    bf16x8_t q[D / 16];
    f32x16_t o[D / 32];
    float m, sum;             // running maximum of the products, and this half's part of the sum
    float ref;                // the maximum, scaled; 0 before a score, and where some row's is past kWide:
    bool wide;                // there the scores' differences from the maximum are scaled
    uint32_t koff[D / 16], voff[D / 32][2];   // byte offsets of the lane's fragment reads in a staged 32-key tile

    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        sum = ref = 0.f;
        wide = false;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    }
    __device__ __forceinline__ void offsets(int lane) {
        constexpr int ROWB = D * 2, CPR = D / 8;
        const int ln = lane & 31, hf = lane >> 5, g2 = (lane >> 4) & 1, i16 = lane & 15;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            koff[j] = (uint32_t)(ln * ROWB + (((2 * j + hf) ^ swz<CPR>(ln)) * 16));
            asm volatile("" : "+v"(koff[j]));
        }
        const int vrow = 4 * hf + (i16 >> 2);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int chunk = 4 * dt + 2 * g2 + ((i16 & 3) >> 1), r = vrow + 8 * x;
                voff[dt][x] = (uint32_t)(r * ROWB + ((chunk ^ swz<CPR>(r)) * 16) + (i16 & 1) * 8);
                asm volatile("" : "+v"(voff[dt][x]));
            }
    }
    // the row's queries; a negative logit scale moves into them (exact in bf16), so that maxima can be taken on the products
    __device__ __forceinline__ void load_q(const unsigned char* row, int hf, bool negative) {
        const uint32_t sgn = negative ? 0x80008000u : 0u;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            uint4 t = *(const uint4*)(row + 32 * j + 16 * hf);
            t.x ^= sgn; t.y ^= sgn; t.z ^= sgn; t.w ^= sgn;
            q[j] = __builtin_bit_cast(bf16x8_t, t);
        }
    }

    // NKT tiles of 32 staged keys.  MASKED: the row sees the keys up to `lim` (of the stage), bit x of `bad` hides keys
    // 16x ... 16x+15, tiles from `tiles` on are seen by no row of the wavefront, those in front of `full` by all of them.  The
    // probabilities are rounded to bf16 (the product's operand) against the maximum up to the end of these tiles, as in the prompt
    // attention of rectangular batches; their sum is of the unrounded ones, in fp32.  SPLIT: each is the sum of two bf16 numbers, 16 bits
    // in all, for twice the second products, which a stream of keys that HBM bounds hides.
    template <int NKT, bool MASKED, bool SPLIT = false>
    __device__ __forceinline__ void attend(const unsigned char* sK, const unsigned char* sV, float qs, int lane, int lim, uint32_t bad,
                                           int tiles, int full) {
        constexpr int ROWB = D * 2, NJ = D / 16, NDT = D / 32, CPR = D / 8;
        const int hf = lane >> 5;
        f32x16_t s[NKT];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) {
                const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sK + kt * 32 * ROWB + koff[j]));
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[j], s[kt], 0, 0, 0);
            }
        // Six fragments ahead (4 to 11 are within the spread of 1 %); left to itself the compiler reads one, waits for it and multiplies.  (Two
        // tiles' products in turn have no wait for each other either.  680 rows, H32: 21.6 us -> 19.9.  The exponentials of one tile
        // spread between the products of the other by the same means, in this order or a tile at a time, gave nothing or cost 4 %.)
        constexpr int kFrags = NKT * NJ, kEarly = kFrags < 6 ? kFrags : 6;
        __builtin_amdgcn_sched_group_barrier(0x100, kEarly, 0);
#pragma unroll
        for (int i = 0; i < kFrags - kEarly; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kEarly, 0);
        if constexpr (MASKED) {
            const int mine = lim - 4 * hf;                    // register r holds key 8 (r/4) + r%4 + 4 hf
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 32 * kt + 8 * (r >> 2) + (r & 3) <= mine ? s[kt][r] : -INFINITY;
            if (bad != 0) {
#pragma unroll
                for (int x = 0; x < 2 * NKT; ++x)
                    if ((bad >> x) & 1u) {
#pragma unroll
                        for (int r = 0; r < 8; ++r) s[x / 2][8 * (x % 2) + r] = -INFINITY;
                    }
            }
        }
        float mx[NKT];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
            mx[kt] = s[kt][0];
#pragma unroll
            for (int r = 1; r + 1 < 16; r += 2) mx[kt] = fmaxf(fmaxf(mx[kt], s[kt][r]), s[kt][r + 1]);
            mx[kt] = fmaxf(mx[kt], s[kt][15]);
        }
        float top = mx[0], corr = 1.f;
#pragma unroll
        for (int kt = 1; kt < NKT; ++kt) top = fmaxf(top, mx[kt]);
        // most stages of a long prompt move no row's maximum: one look, before the two halves of a row exchange theirs
        if (__builtin_amdgcn_ballot_w64(top > m)) {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            const float next = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
            corr = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - next) * qs);
            m = next;
            ref = m == -INFINITY ? 0.f : m * qs;
            wide = __builtin_amdgcn_ballot_w64(fabsf(ref) > kWide) != 0;
            ref = wide ? 0.f : ref;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= corr;
        }
        // One fma scales a score and takes the maximum from it; up to kWide its half step is below 2^-13 and the same for a whole row.
        if (__builtin_expect(wide, 0)) {
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] -= base;
        }
        sum *= corr;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
            if (MASKED && kt >= tiles) break;
            bf16x8_t pf[2], rest[2];
            float psum = 0.f;
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
                uint32_t pk[4], rk[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kt][8 * sl + e], qs, -ref));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kt][8 * sl + e + 1], qs, -ref));
                    psum += p0 + p1;
                    if constexpr (SPLIT) {
                        // The upper part is the bf16 number below p and not the nearest, the rest above 0: an infinite value, times
                        // both, stays one.  (0 has two zeros: a key that is not seen adds nothing.)
                        const uint32_t u0 = __builtin_elementwise_sub_sat(__float_as_uint(p0), 1u) & 0xffff0000u;
                        const uint32_t u1 = __builtin_elementwise_sub_sat(__float_as_uint(p1), 1u) & 0xffff0000u;
                        pk[e / 2] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
                        rk[e / 2] = pack_bf16(p0 - __uint_as_float(u0), p1 - __uint_as_float(u1));
                    } else {
                        pk[e / 2] = pack_bf16(p0, p1);
                    }
                    if constexpr (MASKED) { s[kt][8 * sl + e] = p0; s[kt][8 * sl + e + 1] = p1; }
                }
                pf[sl] = __builtin_bit_cast(bf16x8_t, make_uint4(pk[0], pk[1], pk[2], pk[3]));
                if constexpr (SPLIT) rest[sl] = __builtin_bit_cast(bf16x8_t, make_uint4(rk[0], rk[1], rk[2], rk[3]));
            }
            sum += psum;
            if constexpr (MASKED) {
                // An infinite or NaN value that some rows must not see would reach them as 0 * value: such a tile is added up row by
                // row, over the keys that each of them sees.  (Looked for where a row may not see a key.  It takes 1.5 us
                // of a prompt of 680 rows, H32, 20 us; a look at the copies in front of the barrier, a quarter each, took 2.5, and
                // working a tile over again whose output is not finite more than that in spilled registers.)
                if (kt >= full && wild_values<32 * ROWB / 1024>(sV + 32 * kt * ROWB, lane)) {
                    const int ln = lane & 31;
#pragma unroll 1
                    for (int r = 0; r < 16; ++r) {
                        const float w = s[kt][0];
                        // the registers move on by one: an index that a loop counts would put them into memory
#pragma unroll
                        for (int x = 0; x < 15; ++x) s[kt][x] = s[kt][x + 1];
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) {
                            const int key = 32 * kt + 8 * (r >> 2) + (r & 3) + 4 * half;
                            const float pw = __shfl(w, ln + 32 * half, kWave);
                            const bool see = key <= lim && !((bad >> (key >> 4)) & 1u);
#pragma unroll
                            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const uint2 v = *(const uint2*)(sV + key * ROWB + (((4 * dt + c) ^ swz<CPR>(key)) * 16) + 8 * hf);
                                    const float f[4] = {__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
                                                        __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
#pragma unroll
                                    for (int e = 0; e < 4; ++e) o[dt][4 * c + e] = see ? fmaf(pw, f[e], o[dt][4 * c + e]) : o[dt][4 * c + e];
                                }
                        }
                    }
                    continue;
                }
            }
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
                const unsigned char* sVs = sV + (32 * kt + 16 * sl) * ROWB;
                bf16x8_t vf[NDT];
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const v4i16_t a0 = lds_read_tr(sVs + voff[dt][0]), a1 = lds_read_tr(sVs + voff[dt][1]);
                    vf[dt] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt], pf[sl], o[dt], 0, 0, 0);
                }
                if constexpr (SPLIT) {
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt], rest[sl], o[dt], 0, 0, 0);
                }
            }
            if constexpr (MASKED && !SPLIT) {          // (nothing else is left to hide the reads' way: 29.3 us -> 28.9 for six short prompts)
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * NDT, 0);
#pragma unroll
                for (int i = 0; i < NDT; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, NDT, 0);
            }
        }
    }

    // the whole row sum, in both halves
    __device__ __forceinline__ float total() const { return sum + __shfl_xor(sum, 32, kWave); }

    // the finished row
    __device__ __forceinline__ void store(unsigned char* row, int hf, float inv, bool real) const {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) store_columns(o[dt], row + 64 * dt, hf, inv, real);
    }
    // the 32 rows unfinished, as the registers are: numerators, and {maximum, sum} of the halves' rows
    __device__ __forceinline__ void store_tile(float* to, float2* ms, int lane, float all) const {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *(float4*)(to + ((dt * 4 + c) * kWave + lane) * 4) = make_float4(o[dt][4 * c], o[dt][4 * c + 1], o[dt][4 * c + 2], o[dt][4 * c + 3]);
        ms[lane] = make_float2(m, all);
    }
    // the unfinished row: numerators, and {maximum, sum}
    __device__ __forceinline__ void store_part(float* row, float2* ms, int hf, float all) const {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                *(float4*)(row + 32 * dt + 8 * c + 4 * hf) = make_float4(o[dt][4 * c], o[dt][4 * c + 1], o[dt][4 * c + 2], o[dt][4 * c + 3]);
        if (hf == 0) *ms = make_float2(m, all);
    }
};

// What a row of a tile or unit is: row = token * grp + head of the KV head
struct RowAt { int token, head; };
__device__ __forceinline__ RowAt row_at(int row, FastDiv grp) {
    const DivMod x = div_mod(row, grp);
    return {x.q, x.r};
}

// What both kernels share out: segments (sequence, layer of the call), the KV heads of each one after the other.
struct Work {
    PackedParams a;
    FastDiv grp, by_layers;
    int segs;                       // S * L
};
struct Segment { int s, l, first, n, rows, len, before, end; };   // rows: of this call, times the heads of a KV head; keys; keys in front
                                                                  // of the first new row (below 0: the first rows see nothing); keys that some row sees (none without rows)

template <bool PAGED>
__device__ __forceinline__ Segment segment(const Work& p, int i) {
    Segment x;
    const DivMod sl = div_mod(i, p.by_layers);
    x.s = sl.q; x.l = sl.r;
    const int last = p.a.row_off[x.s + 1];
    x.first = p.a.row_off[x.s];
    x.n = new_rows(x.first, last, p.a.T);
    x.len = PAGED ? entries(p.a, x.s, x.l) : x.n;
    const int rows = PAGED ? min(x.n, p.a.max_rows) : x.n;
    x.rows = rows * p.a.grp;
    x.before = x.len - x.n;
    x.end = keys_seen(rows, x.n, x.len);
    return x;
}
template <bool PAGED>
__device__ __forceinline__ Segment uniform_segment(const Work& p, int i) {
    Segment x = segment<PAGED>(p, i);
    x.s = __builtin_amdgcn_readfirstlane(x.s); x.l = __builtin_amdgcn_readfirstlane(x.l);
    x.first = __builtin_amdgcn_readfirstlane(x.first); x.n = __builtin_amdgcn_readfirstlane(x.n);
    x.rows = __builtin_amdgcn_readfirstlane(x.rows); x.len = __builtin_amdgcn_readfirstlane(x.len);
    x.before = __builtin_amdgcn_readfirstlane(x.before); x.end = __builtin_amdgcn_readfirstlane(x.end);
    return x;
}
__device__ __forceinline__ int64_t shfl_up64(int64_t x, int d) {
    const int lo = __shfl_up((int)(uint32_t)x, d, kWave), hi = __shfl_up((int)(x >> 32), d, kWave);
    return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}
__device__ __forceinline__ int64_t lane64(int64_t x, int j) {
    return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), j) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, j));
}

__device__ __forceinline__ int up(int x, int d) { return __shfl_up(x, d, kWave); }
__device__ __forceinline__ int64_t up(int64_t x, int d) { return shfl_up64(x, d); }
__device__ __forceinline__ int of_lane(int x, int j) { return __builtin_amdgcn_readlane(x, j); }
__device__ __forceinline__ int64_t of_lane(int64_t x, int j) { return lane64(x, j); }

// `count` segments, first + i * step, and their places (of type N).  Up to 64 of them (a layer of 64 sequences) are read once, a lane
// each; beyond, they are read again where they are asked for.
template <bool PAGED, class N, class F>
struct Looked {
    const Work& p;
    int lane, count, first, step;
    F cost;                         // places of a segment
    Segment mine;                   // the segment of this lane
    N upto, all;                    // places of the segments up to that one (of the first 64); of all

    __device__ __forceinline__ Looked(const Work& work, int ln, int n, int from, int by, F f)
        : p(work), lane(ln), count(n), first(from), step(by), cost(f) {
        mine = segment<PAGED>(p, first + min(lane, count - 1) * step);
        upto = lane < count ? cost(mine) : (N)0;
        for (int i = lane + kWave; i < count; i += kWave) upto += cost(segment<PAGED>(p, first + i * step));
        for (int d = 1; d < min(count, kWave); d <<= 1) {
            const N before = up(upto, d);
            if (lane >= d) upto += before;
        }
        all = of_lane(upto, min(count, kWave) - 1);
    }
    // which of them holds place x, the place in it, and what it is
    __device__ __forceinline__ int find(N x, N& in, Segment& sg) const {
        if (count <= kWave) {
            const int j = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > x));
            in = x - (j == 0 ? (N)0 : of_lane(upto, j - 1));
            sg.s = __builtin_amdgcn_readlane(mine.s, j); sg.l = __builtin_amdgcn_readlane(mine.l, j);
            sg.first = __builtin_amdgcn_readlane(mine.first, j); sg.n = __builtin_amdgcn_readlane(mine.n, j);
            sg.rows = __builtin_amdgcn_readlane(mine.rows, j); sg.len = __builtin_amdgcn_readlane(mine.len, j);
            sg.before = __builtin_amdgcn_readlane(mine.before, j); sg.end = __builtin_amdgcn_readlane(mine.end, j);
            return j;
        }
        int j = 0;
        N base = 0;
        for (int c = 0; c < count; c += kWave) {
            const N here = c + lane < count ? cost(segment<PAGED>(p, first + (c + lane) * step)) : (N)0;
            N incl = here;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const N before = up(incl, d);
                if (lane >= d) incl += before;
            }
            const unsigned long long at = __builtin_amdgcn_ballot_w64(base + incl > x);
            if (at != 0) {
                j = c + __builtin_ctzll(at);
                in = x - base - of_lane(incl, j - c) + of_lane(here, j - c);
                break;
            }
            base += of_lane(incl, kWave - 1);
        }
        sg = uniform_segment<PAGED>(p, first + j * step);
        return j;
    }
};

// ---- many rows -----------------------------------------------------------------------------------------
struct TileParams : Work {
    int workgroups;                // that share the launch out; 0: a workgroup per tile
    FastDiv by_hkv, by_heads, by_tiles, by_tail;
    int heads_per_xcd;             // of the call's L * Hkv heads; 0: they do not divide up
    int4* cut;                     // workspace [workgroups]: {segment, head, tile, stage} where a workgroup begins; stage 0: with a whole tile
    float* part_o;                 // [2 * workgroups][4 wavefronts][32 * D], as registers are
    float2* part_ms;               // [2 * workgroups][4 wavefronts][64]
};
constexpr int kStartKeys = 192;     // what the start and the end of a tile cost, in keys
constexpr int kJoinStages = 3;      // what a cut costs: two parts written and read again, and a second start

// Where tiles are cut, every workgroup takes the same share of the launch, wherever that begins and ends: tiles differ in length by two
// orders of magnitude (a prompt's first and last one, caches of other layers), and a launch of a workgroup per tile ends with a few
// long ones on an empty chip.  (600 rows over 6000 keys among shorter sequences, H32/8: 135 us so, 108 in
// equal shares, of which 10 join the parts.)
// A tile's cost is the keys that it sees, if it were full, and kStartKeys, in units of one key and row of grp; that has a closed sum.
template <bool PAGED>
struct TileCost {
    int64_t first;                  // of tile 0, without its rows
    int tiles;
    __device__ __forceinline__ TileCost(const Work& p, const Segment& x)
        : first((int64_t)p.a.grp * (max(x.before, 0) + kStartKeys)), tiles((x.rows + kTileRows - 1) / kTileRows) {}
    __device__ __forceinline__ int64_t up_to(int i) const { return i * first + (int64_t)(kTileRows / 2) * i * (i + 1); }   // tiles 0 ... i-1
    __device__ __forceinline__ int64_t of(int i) const { return first + (int64_t)kTileRows * (i + 1); }
};
// stages of tile i
__device__ __forceinline__ int tile_end(const Work& p, const Segment& x, int i) {       // keys that its rows see
    const int last = __builtin_amdgcn_readfirstlane(row_at(min(x.rows, (i + 1) * kTileRows) - 1, p.grp).token);
    return max(0, min(x.len, x.before + last + 1));
}

struct Cut { int seg, head, tile, stage; };

// What the workgroups share out.
template <bool PAGED, class L>
struct Shares {
    const TileParams& p;
    const L& segs;
    int64_t share;                  // places of a workgroup

    __device__ __forceinline__ Shares(const TileParams& params, const L& looked) : p(params), segs(looked) {
        int longest = segs.mine.end;
        for (int i = segs.lane + kWave; i < p.segs; i += kWave) longest = max(longest, segment<PAGED>(p, i).end);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) longest = max(longest, __shfl_xor(longest, d, kWave));
        // where a launch is small a long tile is cut into pieces of eight stages at least
        const int least = min(8, __builtin_amdgcn_readfirstlane(longest) / (2 * kStage) + 1);
        share = max((int64_t)least * kStage * p.a.grp, (int64_t)((double)segs.all / (double)p.workgroups) + 1);
    }
    // Where workgroup w begins.  A cut close to an end of a tile moves there.
    __device__ __forceinline__ Cut cut(int w) const {
        const int64_t x = w * share;
        if (x >= segs.all) return {p.segs, 0, 0, 0};
        int64_t in;
        Cut c;
        Segment sg;
        c.seg = segs.find(x, in, sg);
        const TileCost<PAGED> t(p, sg);
        const int64_t head = t.up_to(t.tiles);
        c.head = min(p.a.Hkv - 1, (int)((double)in / (double)head));       // (a quotient that is rounded up is corrected)
        in -= c.head * head;
        if (in < 0) { --c.head; in += head; }
        int lo = 0, hi = t.tiles;                           // up_to(lo) <= in < up_to(hi)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (t.up_to(mid) <= in) lo = mid; else hi = mid;
        }
        c.tile = lo;
        const int nst = (tile_end(p, sg, lo) + kStage - 1) / kStage;
        c.stage = min(nst, (int)((float)(in - t.up_to(lo)) / (float)t.of(lo) * (float)nst));
        if (c.stage <= kJoinStages && 2 * c.stage <= nst) c.stage = 0;
        else if (nst - c.stage <= kJoinStages) {                    // the next tile
            c.stage = 0;
            if (++c.tile == t.tiles) {
                c.tile = 0;
                if (++c.head == p.a.Hkv) { c.head = 0; ++c.seg; }      // (a segment without tiles is passed over)
            }
        }
        return c;
    }
};
// (the compiler does not see that all lanes agree)
__device__ __forceinline__ Cut uniform(const Cut& c) {
    return {__builtin_amdgcn_readfirstlane(c.seg), __builtin_amdgcn_readfirstlane(c.head), __builtin_amdgcn_readfirstlane(c.tile),
            __builtin_amdgcn_readfirstlane(c.stage)};
}

// A workgroup per tile, where there are many: which one it has.  With heads in eighths every head stays on one XCD: the tiles of a
// head run next to each other and read its keys at about the same time through that XCD's L2; the last heads of an XCD are taken
// together, so that the launch does not end on the long tiles of a single one.  Else heads alternate.  Within a head: sequence by
// sequence, the last tile first, whose rows see the most.
template <bool PAGED>
__device__ __forceinline__ Cut tile_of(const TileParams& p, int lane, int bid, Segment& sg) {
    int head, tt;
    if (p.heads_per_xcd > 0) {
        const int xcd = bid % kXcds, j = bid / kXcds, hx = p.heads_per_xcd, lead = hx - (int)p.by_tail.d, tiles = (int)p.by_tiles.d;
        const bool front = j < lead * tiles;
        const DivMod x = front ? uniform_div_mod(j, p.by_tiles) : uniform_div_mod(j - lead * tiles, p.by_tail);
        head = xcd * hx + (front ? x.q : lead + x.r);
        tt = front ? x.r : x.q;
    } else {
        const DivMod x = uniform_div_mod(bid, p.by_heads);
        head = x.r; tt = x.q;
    }
    const DivMod lg = uniform_div_mod(head, p.by_hkv);
    auto tiles = [&](const Segment& x) { return (x.rows + kTileRows - 1) / kTileRows; };
    const Looked<PAGED, int, decltype(tiles)> looked(p, lane, p.a.S, lg.q, p.a.L, tiles);      // the layer's sequences
    if (tt >= looked.all) return {p.segs, 0, 0, 0};
    int in;
    const int s = looked.find(tt, in, sg);
    return {s * p.a.L + lg.q, lg.r, in, 0};
}

template <int D, bool PAGED, bool WHOLE>
__global__ void __launch_bounds__(256, 2)
attn_tiles_kernel(TileParams p) {
    constexpr int ROWB = D * 2, kInst = CopyLane<D>::kCopies;               // copies per wavefront, stage and tensor: 16 rows
    __shared__ __attribute__((aligned(1024))) unsigned char sKa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sKb[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVb[kStage * ROWB];
    const PackedParams& a = p.a;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int ln = lane & 31, hf = lane >> 5;
    int wg = 0;
    Cut from, to;
    Segment sg;
    if constexpr (WHOLE) {
        from = to = uniform(tile_of<PAGED>(p, lane, (int)blockIdx.x, sg));
    } else {
        // neighbours in the order of the work run on one XCD and share keys through its L2
        wg = (int)xcd_swizzle(blockIdx.x, (uint32_t)p.workgroups);
        auto cost = [&](const Segment& x) {
            const TileCost<PAGED> t(p, x);
            return t.up_to(t.tiles) * a.Hkv;
        };
        const Looked<PAGED, int64_t, decltype(cost)> looked(p, lane, p.segs, 0, 1, cost);
        const Shares<PAGED, decltype(looked)> sh(p, looked);
        from = uniform(sh.cut(wg));
        to = uniform(sh.cut(wg + 1));
        if (threadIdx.x == 0) p.cut[wg] = make_int4(from.seg, from.head, from.tile, from.stage);
    }

    const CopyLane<D> cp(lane);
    RowTile<D> tl;
    tl.offsets(lane);
    int seg = from.seg, g = from.head, tile = from.tile, stage = from.stage;
    while (seg < p.segs && seg <= to.seg) {                 // (`to` may be a segment without rows)
        if constexpr (!WHOLE) sg = uniform_segment<PAGED>(p, seg);
        const int tiles = (sg.rows + kTileRows - 1) / kTileRows;
        if (!WHOLE && tile >= tiles) { tile = 0; g = 0; ++seg; continue; }  // a segment without rows
        if constexpr (WHOLE) tile = tiles - 1 - tile;
        const bool last = !WHOLE && seg == to.seg && g == to.head && tile == to.tile;
        if (last && to.stage == 0) break;
        const int end = tile_end(p, sg, tile), nst = (end + kStage - 1) / kStage;
        const int st0 = stage, st1 = last ? to.stage : nst;

        // this wavefront's rows
        const int r0 = tile * kTileRows + wv * 32, row = r0 + ln;
        const bool mine = r0 < sg.rows, real = row < sg.rows;
        const RowAt ra = row_at(real ? row : mine ? r0 : 0, p.grp);         // (rows that do not exist repeat one that does)
        const int lim = sg.before + ra.token;                               // the last key that the row sees
        const int lim_first = sg.before + __builtin_amdgcn_readfirstlane(row_at(mine ? r0 : 0, p.grp).token);
        const int lim_last = sg.before + __builtin_amdgcn_readfirstlane(row_at(max(min(sg.rows, r0 + 32) - 1, 0), p.grp).token);
        const int h = g * a.grp + ra.head;
        const int64_t t = sg.first + ra.token;

        // Keys and values of a stage: a wavefront copies 16 rows of each, which lie in one page.
        const unsigned char *kb = a.k, *vb = a.v;
        const int32_t* pages = nullptr;
        if constexpr (PAGED) {
            pages = a.table + ((int64_t)sg.s * a.layers + a.l0 + sg.l) * a.max_pages;
        } else {
            kb += a.ks.l * sg.l + a.ks.h * g + a.ks.n * sg.first;
            vb += a.vs.l * sg.l + a.vs.h * g + a.vs.n * sg.first;
        }
        // Page ids ahead of their use: lane i has that of the i-th group of 16 keys from ids0 on, `next` the 64 groups behind them.
        // Ids outside the pool are read as page 0; a tile that has one is worked on with masks throughout.
        int ids = 0, next = 0, ids0 = st0 * 4;
        unsigned long long bad_now = 0, bad_next = 0;
        bool hidden = false;
        auto load_ids = [&](int group) {
            const int key = min((group + lane) * 16, max(end - 1, 0));
            return end > 0 ? pages[key >> a.shift] : 0;
        };
        auto check_ids = [&](int& x) {
            const bool out = (uint32_t)x >= (uint32_t)a.num_pages;
            if (out) x = 0;
            return __builtin_amdgcn_ballot_w64(out);
        };
        if constexpr (PAGED) {
            ids = load_ids(ids0);
            next = load_ids(ids0 + kWave);
            const int to_page = (min(st1 * kStage, end) - 1) >> a.shift;
            for (int i = ((st0 * kStage) >> a.shift) + lane; i <= to_page; i += kWave) hidden = hidden || (uint32_t)pages[i] >= (uint32_t)a.num_pages;
            hidden = __builtin_amdgcn_ballot_w64(hidden) != 0;
            bad_now = check_ids(ids);
            bad_next = check_ids(next);
        }
        auto issue = [&](int st, unsigned char* dK, unsigned char* dV) -> uint32_t {
            uint32_t bad = 0;
            const int key = min(st * kStage + wv * 16, end - 1);            // the group's first key, or the last one there is
            const uint32_t rest = (uint32_t)(end - 1 - key);
            if constexpr (PAGED) {
                if (st * 4 >= ids0 + kWave) {
                    ids = next; bad_now = bad_next; ids0 += kWave;
                    next = load_ids(ids0 + kWave);
                    bad_next = check_ids(next);
                }
                bad = (uint32_t)((bad_now >> (st * 4 - ids0)) & 15u);
                const int64_t id = __builtin_amdgcn_readlane(ids, st * 4 + wv - ids0);
                const int64_t base = (((id * a.Hkv + g) << a.shift) + (key & ((1 << a.shift) - 1))) * ROWB;
#pragma unroll
                for (int i = 0; i < kInst; ++i) {
                    const uint32_t off = cp.at(i, rest, ROWB);
                    copy_to_lds(kb + base + off, dK + (wv * kInst + i) * 1024);
                    copy_to_lds(vb + base + off, dV + (wv * kInst + i) * 1024);
                }
            } else {
                const unsigned char *ka = kb + a.ks.n * (int64_t)key, *va = vb + a.vs.n * (int64_t)key;
#pragma unroll
                for (int i = 0; i < kInst; ++i) {
                    copy_to_lds(ka + cp.at(i, rest, (uint32_t)a.ks.n), dK + (wv * kInst + i) * 1024);
                    copy_to_lds(va + cp.at(i, rest, (uint32_t)a.vs.n), dV + (wv * kInst + i) * 1024);
                }
            }
            return bad;
        };
        uint32_t bad_a = 0, bad_b = 0;
        const int seen = sg.before + __builtin_amdgcn_readfirstlane(row_at(tile * kTileRows, p.grp).token) + 1;
        const int plain = hidden ? 0 : max(0, min(st1, seen / kStage) - st0);
        if (st0 < st1) {
            if (plain & 1) issue(st0, sKb, sVb);
            else bad_a = issue(st0, sKa, sVa);
        }

        const float sc = a.scale[sg.l], qs = score_scale(sc), size = scale_size(sc);
        tl.load_q(a.q + a.qs.l * sg.l + a.qs.h * h + a.qs.n * t, hf, sc < 0.f);
        tl.clear();

        auto sync = [&]() {
            __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wavefront's part of the stage has landed
            __syncthreads();                                     // ... and everybody's; the other pair is free again
        };
        // Stages whose keys every row of the tile sees, two at a time, without a branch between them: a masked stage in the same
        // loop made the compiler move the output between two sets of registers (four prompts of 8192 rows then 3160 us, so 2870).  A
        // wavefront without rows works along on rows that are not stored.
        int st = st0;
        if (plain & 1) {                                         // (the first stage of an odd number is in the other pair)
            sync();
            if (st + 1 < st1) bad_a = issue(st + 1, sKa, sVa);
            tl.template attend<2, false>(sKb, sVb, qs, lane, 0, 0u, 2, 2);
            ++st;
        }
        for (; st < st0 + plain; st += 2) {
            sync();
            issue(st + 1, sKb, sVb);
            tl.template attend<2, false>(sKa, sVa, qs, lane, 0, 0u, 2, 2);
            sync();
            if (st + 2 < st1) bad_a = issue(st + 2, sKa, sVa);
            tl.template attend<2, false>(sKb, sVb, qs, lane, 0, 0u, 2, 2);
        }
        auto attend = [&](int st, const unsigned char* sK, const unsigned char* sV, uint32_t bad) {
            const int key0 = st * kStage;
            if (mine && key0 <= lim_last)
                tl.template attend<2, true>(sK, sV, qs, lane, lim - key0, bad, key0 + 32 <= lim_last ? 2 : 1,
                                            bad != 0 ? 0 : (max(lim_first - key0, -1) + 1) / 32);
        };
        for (; st < st1; st += 2) {
            sync();
            if (st + 1 < st1) bad_b = issue(st + 1, sKb, sVb);
            attend(st, sKa, sVa, bad_a);
            if (st + 1 >= st1) break;
            sync();
            if (st + 2 < st1) bad_a = issue(st + 2, sKa, sVa);
            attend(st + 1, sKb, sVb, bad_b);
        }
        if (mine) {
            const float sum = tl.total();
            if (WHOLE || (st0 == 0 && st1 == nst)) {
                tl.store(a.out + a.os.l * sg.l + a.os.h * h + a.os.n * t, hf, sum == 0.f ? 0.f : 1.f / sum, real);
                if (!PAGED && real && hf == 0)
                    a.lse[(int64_t)a.L * a.H * sg.first + (int64_t)(sg.l * a.H + h) * sg.n + ra.token] = fmaf(tl.m, size, kLn2 * __builtin_amdgcn_logf(sum));
            } else {
                // a workgroup has at most two parts of tiles that others share: of one that began before it, and of one that goes on
                const int64_t slot = (int64_t)(2 * wg + (st0 > 0 ? 0 : 1)) * 4 + wv;
                tl.store_tile(p.part_o + slot * 32 * D, p.part_ms + slot * kWave, lane, sum);
            }
        }
        if (WHOLE || last) break;
        stage = 0;
        if (++tile == tiles) {
            tile = 0;
            if (++g == a.Hkv) { g = 0; ++seg; }
        }
        __syncthreads();                                         // the buffers are free
    }
}

// Joins the parts of the tiles that were cut: the first cut of a tile has all of its parts.  A wavefront has 32 columns of 32 rows, in
// the registers' order, in which the parts were written.  Bound: reading the parts, two of 64 KB for each workgroup at most at D 128;
// 9.6 us for 512 workgroups.
template <int D, bool PAGED>
__global__ void __launch_bounds__(kWave)
attn_merge_tiles_kernel(TileParams p) {
    const PackedParams& a = p.a;
    const int w0 = (int)blockIdx.x + 1, lane = threadIdx.x, wv = (int)blockIdx.y / (D / 32), dt = (int)blockIdx.y % (D / 32);
    const int ln = lane & 31, hf = lane >> 5;
    // the cuts from the one before this on: those inside the same tile follow each other
    int w1 = w0;
    int4 c;
    for (int base = w0 - 1;; base += kWave) {
        const int4 x = p.cut[min(base + lane, p.workgroups - 1)];
        if (base == w0 - 1) {
            c = make_int4(__builtin_amdgcn_readlane(x.x, 1), __builtin_amdgcn_readlane(x.y, 1), __builtin_amdgcn_readlane(x.z, 1),
                          __builtin_amdgcn_readlane(x.w, 1));
            if (c.w == 0) return;
        }
        const bool same = base + lane < p.workgroups && x.w != 0 && x.x == c.x && x.y == c.y && x.z == c.z;
        unsigned long long m = __builtin_amdgcn_ballot_w64(same);
        if (base == w0 - 1) {
            if (m & 1ull) return;                                // a later cut of its tile
            m |= 1ull;
        }
        const int run = ~m == 0ull ? kWave : __builtin_ctzll(~m);
        w1 = base + run - 1;
        if (run < kWave) break;
    }
    const Segment sg = uniform_segment<PAGED>(p, c.x);
    const int r0 = c.z * kTileRows + wv * 32, row = r0 + ln;
    if (r0 >= sg.rows) return;
    const float size = scale_size(a.scale[sg.l]), qs = size * kLog2e;
    float m = -INFINITY, sum = 0.f;
    f32x16_t o;
#pragma unroll
    for (int r = 0; r < 16; ++r) o[r] = 0.f;
#pragma unroll 4
    for (int w = w0 - 1; w <= w1; ++w) {                         // a running maximum: every part is read once
        const int64_t slot = (int64_t)(2 * w + (w < w0 ? 1 : 0)) * 4 + wv;
        const float2 x = p.part_ms[slot * kWave + lane];
        const float4* from = (const float4*)(p.part_o + slot * 32 * D) + dt * 4 * kWave + lane;
        const float4 y[4] = {from[0], from[kWave], from[2 * kWave], from[3 * kWave]};
        const float mx = fmaxf(m, x.x), ref = mx == -INFINITY ? 0.f : mx;
        const float c0 = __builtin_amdgcn_exp2f((m - ref) * qs), c1 = __builtin_amdgcn_exp2f((x.x - ref) * qs);
        sum = fmaf(sum, c0, x.y * c1);
        m = mx;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            o[4 * i] = fmaf(o[4 * i], c0, y[i].x * c1); o[4 * i + 1] = fmaf(o[4 * i + 1], c0, y[i].y * c1);
            o[4 * i + 2] = fmaf(o[4 * i + 2], c0, y[i].z * c1); o[4 * i + 3] = fmaf(o[4 * i + 3], c0, y[i].w * c1);
        }
    }
    const bool real = row < sg.rows;
    const RowAt ra = row_at(real ? row : r0, p.grp);
    const int h = c.y * a.grp + ra.head;
    store_columns(o, a.out + a.os.l * sg.l + a.os.h * h + a.os.n * (int64_t)(sg.first + ra.token) + 64 * dt, hf, sum == 0.f ? 0.f : 1.f / sum, real);
    if (!PAGED && real && hf == 0 && dt == 0)
        a.lse[(int64_t)a.L * a.H * sg.first + (int64_t)(sg.l * a.H + h) * sg.n + ra.token] = fmaf(m, size, kLn2 * __builtin_amdgcn_logf(sum));
}

// ---- few rows: the keys of a launch shared out evenly over the wavefronts ---------------------------------
struct StreamParams : Work {
    int waves;
    int join_rows;                  // rows of a workgroup that joins: 1, or all of its groups of lanes
    int* share;                     // workspace: blocks of a wavefront
    int* start;                     // [segs]: first block of a segment (segments that have blocks)
    float* part_o;                  // [2 * waves][32][D]
    float2* part_ms;
};
constexpr int kLeastBlocks = 2;     // of a wavefront

__device__ __forceinline__ int blocks_of(const Segment& x) { return (x.end + kBlockKeys - 1) / kBlockKeys; }

template <int D>
__global__ void __launch_bounds__(128, 128 / D)
attn_stream_kernel(StreamParams p) {
    constexpr int ROWB = D * 2, kBytes = kBlockKeys * ROWB, kInst = CopyLane<D>::kCopies;            // copies per 16 keys and tensor
    __shared__ __attribute__((aligned(1024))) unsigned char sKa[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sVa[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sKb[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sVb[2][kBytes];
    const PackedParams& a = p.a;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 2 + wv), ln = lane & 31, hf = lane >> 5;

    // the launch's blocks, and this wavefront's: segment by segment, KV head by KV head
    auto blocks = [&](const Segment& x) { return (int64_t)blocks_of(x) * a.Hkv; };
    const Looked<true, int64_t, decltype(blocks)> looked(p, lane, p.segs, 0, 1, blocks);
    const int all_blocks = (int)looked.all;                                // (below 2^31: the call is refused otherwise)
    const int share = max(kLeastBlocks, (all_blocks + p.waves - 1) / p.waves);
    if (wave == 0 && lane == 0) *p.share = share;
    const int b0 = (int)min((int64_t)wave * share, (int64_t)all_blocks), b1 = (int)min((int64_t)b0 + share, (int64_t)all_blocks);
    if (b0 >= b1) return;
    int64_t in_seg;
    Segment sg;
    const int seg = looked.find(b0, in_seg, sg);

    // where copies are asked for (`in`), and where the work is (`sg`): both walk the same blocks
    struct Cursor { int seg, g, blk; };
    Segment in = sg;
    Cursor cw = {seg, 0, (int)in_seg};
    cw.g = cw.blk / blocks_of(sg);
    cw.blk -= cw.g * blocks_of(sg);
    int seg_start = b0 - (int)in_seg;                           // first block of the segment worked on
    Cursor ci = cw;
    auto step = [&](Cursor& c, Segment& x) -> bool {            // true: another segment
        if (++c.blk < blocks_of(x)) return false;
        c.blk = 0;
        if (++c.g < a.Hkv) return false;
        c.g = 0;
        do { ++c.seg; x = uniform_segment<true>(p, c.seg); } while (x.end == 0);    // (a block is left, so a segment is)
        return true;
    };
    const CopyLane<D> cp(lane);
    // lane i has the page of the i-th group of 16 keys from ids0 on
    int ids = 0, ids0 = 0;
    unsigned long long bad_ids = 0;
    auto load_ids = [&]() {
        const int32_t* pages = a.table + ((int64_t)in.s * a.layers + a.l0 + in.l) * a.max_pages;
        ids0 = 2 * ci.blk;
        ids = pages[min((ids0 + lane) * 16, in.end - 1) >> a.shift];
        const bool out = (uint32_t)ids >= (uint32_t)a.num_pages;
        if (out) ids = 0;
        bad_ids = __builtin_amdgcn_ballot_w64(out);
    };
    load_ids();
    auto issue = [&](unsigned char* dK, unsigned char* dV) -> uint32_t {
        const uint32_t bad = (uint32_t)((bad_ids >> (2 * ci.blk - ids0)) & 3u);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t id = __builtin_amdgcn_readlane(ids, 2 * ci.blk + x - ids0);
            const int key = min(ci.blk * kBlockKeys + 16 * x, in.end - 1);
            const int64_t base = (((id * a.Hkv + ci.g) << a.shift) + (key & ((1 << a.shift) - 1))) * ROWB;
            const uint32_t last = (uint32_t)(in.end - 1 - key);
#pragma unroll
            for (int i = 0; i < kInst; ++i) {
                const uint32_t off = cp.at(i, last, ROWB);
                copy_to_lds(a.k + base + off, dK + (x * kInst + i) * 1024);
                copy_to_lds(a.v + base + off, dV + (x * kInst + i) * 1024);
            }
        }
        return bad;
    };
    // moves on to the next block, if there is one, and asks for it
    int asked = b0;
    auto ask = [&](unsigned char* dK, unsigned char* dV) -> uint32_t {
        if (asked > b0) {
            const bool other = step(ci, in);
            if (other || 2 * ci.blk + 1 >= ids0 + kWave || 2 * ci.blk < ids0) load_ids();
        }
        ++asked;
        return issue(dK, dV);
    };

    RowTile<D> tl;
    tl.offsets(lane);
    float qs = 1.f;
    int lim = 0, piece = cw.blk;                                // piece: the unit's first block here
    unsigned char* out = nullptr;
    auto begin = [&]() {                                        // a unit: its queries
        const RowAt ra = row_at(ln < sg.rows ? ln : 0, p.grp);
        const int h = cw.g * a.grp + ra.head;
        const int64_t t = sg.first + ra.token;
        const float sc = a.scale[sg.l];
        qs = score_scale(sc);
        tl.load_q(a.q + a.qs.l * sg.l + a.qs.h * h + a.qs.n * t, hf, sc < 0.f);
        out = a.out + a.os.l * sg.l + a.os.h * h + a.os.n * t;
        lim = sg.before + ra.token;
        tl.clear();
        piece = cw.blk;
        if (cw.g == 0 && cw.blk == 0 && lane == 0) p.start[cw.seg] = seg_start;
    };
    auto end = [&](bool whole) {
        const float all = tl.total();
        const bool real = ln < sg.rows;
        if (whole && piece == 0) { tl.store(out, hf, all == 0.f ? 0.f : 1.f / all, real); return; }
        // a wavefront has at most two pieces of units that others share: one that began before it, one that goes on behind it
        const int64_t slot = (int64_t)(2 * wave + (piece == 0 ? 1 : 0)) * kFewRows + ln;
        if (real) tl.store_part(p.part_o + slot * D, p.part_ms + slot, hf, all);
    };
    auto attend = [&](const unsigned char* sK, const unsigned char* sV, uint32_t bad) {
        const int key0 = cw.blk * kBlockKeys;
        if (key0 + kBlockKeys - 1 <= sg.before && bad == 0) tl.template attend<1, false, true>(sK, sV, qs, lane, 0, 0u, 1, 1);
        else tl.template attend<1, true, true>(sK, sV, qs, lane, lim - key0, bad, 1, 0);
    };
    // one block of the work: `more` blocks are in flight behind it
    auto work = [&](int b, const unsigned char* sK, const unsigned char* sV, uint32_t bad) {
        attend(sK, sV, bad);
        const bool whole = cw.blk + 1 == blocks_of(sg);
        if (whole || b + 1 == b1) {
            end(whole);
            if (b + 1 < b1) {
                const int old = blocks_of(sg);
                if (step(cw, sg)) seg_start += old * a.Hkv;
                begin();
            }
        } else {
            ++cw.blk;
        }
    };
    constexpr int kCopies = 4 * kInst;                          // of a block
    uint32_t bad_a = ask(sKa[wv], sVa[wv]), bad_b = 0;
    begin();
    if (asked < b1) bad_b = ask(sKb[wv], sVb[wv]);
    auto landed = [&](int b) {                                  // block b is in LDS; the next one may be on its way
        if (asked > b + 1) {
            if constexpr (kCopies == 16) __builtin_amdgcn_s_waitcnt(0x4F70);    // vmcnt(16)
            else __builtin_amdgcn_s_waitcnt(0x0F78);                           // vmcnt(8)
        } else {
            __builtin_amdgcn_s_waitcnt(0x0F70);
        }
        asm volatile("" ::: "memory");
    };
    for (int b = b0; b < b1; b += 2) {
        landed(b);
        work(b, sKa[wv], sVa[wv], bad_a);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the fragment reads are done: the buffer is free
        if (asked < b1) bad_a = ask(sKa[wv], sVa[wv]);
        if (b + 1 >= b1) break;
        landed(b + 1);
        work(b + 1, sKb[wv], sVb[wv], bad_b);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (asked < b1) bad_b = ask(sKb[wv], sVb[wv]);
    }
}

// Joins the pieces of a unit's rows; rows of units without a block get zeros.  D / 4 lanes have a row.  Units of up to eight rows get a
// workgroup per row, whose groups of lanes share the row's pieces (one sequence of 8192 keys, H32/8: 128 pieces per unit); with more
// rows there are few pieces, and a group has a row (a workgroup per row took 42 us for 1600 units of 20 rows that nobody shared).
constexpr int kJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kJoinThreads)
attn_merge_stream_kernel(StreamParams p) {
    constexpr int LPP = D / 4, GROUPS = kJoinThreads / LPP;
    __shared__ float2 s_ms[GROUPS];
    __shared__ float4 s_o[GROUPS][LPP];
    const PackedParams& a = p.a;
    const int i = (int)blockIdx.x / a.Hkv, g = (int)blockIdx.x % a.Hkv;
    const int share = max(1, *p.share), start = p.start[i];     // (asked for with the segment; `start` is looked at if it has blocks)
    const float qs = score_scale(a.scale[uniform_div_mod(i, p.by_layers).r]);
    const Segment x = uniform_segment<true>(p, i);
    if ((int)blockIdx.y * p.join_rows >= x.rows) return;
    const int u0 = x.end == 0 ? 0 : start + g * blocks_of(x);
    const int w0 = u0 / share, w1 = (u0 + blocks_of(x) - 1) / share;
    if (x.end > 0 && w0 == w1) return;                          // one wavefront has written it
    const int c = threadIdx.x % LPP, group = threadIdx.x / LPP;
    const int rows = p.join_rows, pieces = GROUPS / rows, mine = group / rows;      // rows here, groups of a row, and which this is
    const int row = (int)blockIdx.y * rows + group % rows;
    float m = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row < x.rows && x.end > 0) {
#pragma unroll 4
        for (int w = w0 + mine; w <= w1; w += pieces) {     // a running maximum: every piece is read once
            const int64_t slot = (int64_t)(2 * w + (w == w0 ? 1 : 0)) * kFewRows + row;
            const float2 ms = p.part_ms[slot];
            const float4 y = *(const float4*)(p.part_o + slot * D + 4 * c);
            const float mx = fmaxf(m, ms.x), ref = mx == -INFINITY ? 0.f : mx;
            const float c0 = __builtin_amdgcn_exp2f((m - ref) * qs), c1 = __builtin_amdgcn_exp2f((ms.x - ref) * qs);
            sum = fmaf(sum, c0, ms.y * c1);
            o.x = fmaf(o.x, c0, y.x * c1); o.y = fmaf(o.y, c0, y.y * c1); o.z = fmaf(o.z, c0, y.z * c1); o.w = fmaf(o.w, c0, y.w * c1);
            m = mx;
        }
    }
    if (pieces > 1) {
        if (c == 0) s_ms[group] = make_float2(m, sum);
        s_o[group][c] = o;
        __syncthreads();
        if (mine == 0) {
            float top = m;
            for (int k = 1; k < pieces; ++k) top = fmaxf(top, s_ms[group + k * rows].x);
            const float ref = top == -INFINITY ? 0.f : top, c0 = __builtin_amdgcn_exp2f((m - ref) * qs);
            sum *= c0;
            o.x *= c0; o.y *= c0; o.z *= c0; o.w *= c0;
            for (int k = 1; k < pieces; ++k) {
                const float2 ms = s_ms[group + k * rows];
                const float4 y = s_o[group + k * rows][c];
                const float c1 = __builtin_amdgcn_exp2f((ms.x - ref) * qs);
                sum = fmaf(ms.y, c1, sum);
                o.x = fmaf(y.x, c1, o.x); o.y = fmaf(y.y, c1, o.y); o.z = fmaf(y.z, c1, o.z); o.w = fmaf(y.w, c1, o.w);
            }
        }
    }
    if (mine == 0 && row < x.rows) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const RowAt ra = row_at(row, p.grp);
        const int h = g * a.grp + ra.head;
        *(uint2*)(a.out + a.os.l * x.l + a.os.h * h + a.os.n * (int64_t)(x.first + ra.token) + 8 * c) =
            make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    }
}

// ---- launches ------------------------------------------------------------------------------------------
constexpr int kStreamWorkgroups = 2;          // of a compute unit: 64 KB of LDS each at D = 128
constexpr int kTileWorkgroups = 2;            // of attn_tiles_kernel: 256 registers

constexpr int kTailTiles = 256;               // workgroups of an XCD at the end of a launch whose heads are taken together

static bool few_rows(const pkv_packed& s, int max_rows) { return max_rows > 0 && (int64_t)max_rows * (s.H / s.Hkv) <= kFewRows; }
static int stream_waves(const pkv_packed& s) { return compute_units() * kStreamWorkgroups * 2 * (128 / s.D); }
static int tile_workgroups() { return compute_units() * kTileWorkgroups / kXcds * kXcds; }
static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// tiles of all sequences of a KV head at most
static long long most_tiles(const pkv_packed& s) { return (long long)s.T * (s.H / s.Hkv) / kTileRows + (s.S < s.T ? s.S : s.T); }
// Whether tiles are cut.  A launch of a workgroup per tile takes as long as its longest tile (1.27 us a stage with a compute unit of
// its own) or as the whole work shared out (2.0 us a stage on each of the workgroups), whichever is longer; cutting brings the first down
// to the second and costs about 30 us (parts, joining them, shares, a phase of its own for every workgroup).  The longest tile and the
// average are taken from the most that can be: the rows of a prompt, the width of a table row, of which a cache holds three quarters.
// us, whole / cut: H32/8, 512 rows over 8192 keys 178 / 108, 4 x 128 rows 168 / 104, 16 x 40 over 2000 50 / 59; H32, 8 x 64 over 1000
// 31 / 46, 64 over 4000 80 / 40; one prompt: H32 680 19 / 37, 2048 52 / 69, H8 2048 43 / 38, H12/4 6000 140 / 149.
// What the lengths are is on the device, so the bounds are wide where the rows are several prompts' (T stands for the longest) or the
// table is wider than its caches, and launches are cut that would be faster whole: prompts of H12/4, 6 x 500 21 / 31, H8/2, 12 x 500
// 24 / 32, H4, 16 x 1000 41 / 57, H8/1, 64 x 100 13 / 20; H32/8, 8 x 64 rows over 1000 entries of a table of 8192 27 / 43.
static bool cut_tiles(const pkv_packed& s, long long keys, bool paged) {
    const double stages = (double)((keys + kStage - 1) / kStage), tiles = (double)most_tiles(s) * s.L * s.Hkv;
    return stages * (1.27 - (paged ? 0.75 : 0.5) * 2.0 * tiles / tile_workgroups()) > 30.0;
}

// rows of a KV head and block numbers are 32 bits wide, and so are the threads of a grid (256 of a workgroup)
bool packed_attn_fits(const pkv_packed& s, const pkv_paging* g) {
    if ((int64_t)s.T * (s.H / s.Hkv) > 0x7fffff00ll) return false;
    if ((int64_t)s.S * s.L * s.Hkv >= 1 << 24 || most_tiles(s) * s.L * s.Hkv >= 1 << 24) return false;
    return !g || (double)s.S * s.L * s.Hkv * g->max_pages * g->page_size / kBlockKeys < 2147483648.0;
}

size_t packed_attn_ws_bytes(const pkv_packed& s, int max_rows) {
    if (s.dtype != PKV_BF16) return 0;
    const size_t row = sizeof(float2) + s.D * sizeof(float);                    // (a part of a tile has two of the first per row)
    if (few_rows(s, max_rows)) return 256 + up256((size_t)s.S * s.L * 4) + (size_t)2 * stream_waves(s) * kFewRows * row;
    // (whether tiles are cut goes by the table's width too, which the size does not ask for: where the widest would not be, none is)
    if (!cut_tiles(s, max_rows > 0 ? kMaxSegmentSlots : s.T, max_rows > 0)) return 0;
    return up256(tile_workgroups() * sizeof(int4)) + (size_t)2 * tile_workgroups() * kTileRows * (row + sizeof(float2));
}

static Work work_of(const pkv_packed& s, const PackedParams& a) {
    Work w;
    w.a = a;
    w.grp = fast_div(a.grp); w.by_layers = fast_div(s.L);
    w.segs = s.S * s.L;
    return w;
}

template <int D, bool PAGED>
static hipError_t launch_tiles(const pkv_packed& s, const PackedParams& a, void* ws, hipStream_t st) {
    TileParams p;
    (Work&)p = work_of(s, a);
    const long long tiles = most_tiles(s), heads = (long long)s.L * s.Hkv;
    p.by_hkv = fast_div(s.Hkv); p.by_heads = fast_div(heads); p.by_tiles = fast_div(tiles);
    p.heads_per_xcd = heads % kXcds == 0 ? (int)(heads / kXcds) : 0;
    const long long tail = (kTailTiles + tiles - 1) / tiles;
    p.by_tail = fast_div(tail < p.heads_per_xcd ? tail : p.heads_per_xcd > 0 ? p.heads_per_xcd : 1);
    p.cut = (int4*)ws;
    p.workgroups = tile_workgroups();
    p.part_o = (float*)((char*)ws + up256(p.workgroups * sizeof(int4)));
    p.part_ms = (float2*)(p.part_o + (size_t)2 * p.workgroups * kTileRows * D);
    if (!cut_tiles(s, PAGED ? (long long)a.max_pages << a.shift : s.T, PAGED)) {
        hipLaunchKernelGGL((attn_tiles_kernel<D, PAGED, true>), dim3((unsigned)(tiles * heads)), dim3(256), 0, st, p);
    } else {
        hipLaunchKernelGGL((attn_tiles_kernel<D, PAGED, false>), dim3((unsigned)p.workgroups), dim3(256), 0, st, p);
        hipLaunchKernelGGL((attn_merge_tiles_kernel<D, PAGED>), dim3((unsigned)p.workgroups - 1, kTileRows / 32 * (D / 32)), dim3(kWave), 0,
                           st, p);
    }
    return hipGetLastError();
}

template <int D>
static hipError_t launch_stream(const pkv_packed& s, const PackedParams& a, void* ws, hipStream_t st) {
    StreamParams p;
    (Work&)p = work_of(s, a);
    p.waves = stream_waves(s);
    p.share = (int*)ws;
    p.start = (int*)((char*)ws + 256);
    p.part_o = (float*)((char*)ws + 256 + up256((size_t)p.segs * 4));
    p.part_ms = (float2*)(p.part_o + (size_t)2 * p.waves * kFewRows * D);
    const int rows = a.max_rows * a.grp;
    p.join_rows = rows <= 8 ? 1 : kJoinThreads / (D / 4);
    hipLaunchKernelGGL(attn_stream_kernel<D>, dim3((unsigned)(p.waves / 2)), dim3(128), 0, st, p);
    hipLaunchKernelGGL(attn_merge_stream_kernel<D>, dim3((unsigned)(p.segs * s.Hkv), (unsigned)((rows + p.join_rows - 1) / p.join_rows)),
                       dim3(kJoinThreads), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_packed_attn(const pkv_packed& s, const PackedAttn& a, hipStream_t st) {
    const int esize = s.dtype == PKV_F32 ? 4 : 2;
    auto bytes = [esize](Strides x) { return Strides{0, x.l * esize, x.h * esize, x.n * esize}; };
    PackedParams p;
    p.S = s.S; p.L = s.L; p.H = s.H; p.Hkv = s.Hkv; p.T = s.T; p.grp = s.H / s.Hkv;
    const bool paged = a.table != nullptr;
    p.num_pages = a.g.num_pages; p.max_pages = a.g.max_pages; p.layers = a.g.layers; p.l0 = a.l0; p.max_rows = a.max_rows;
    p.shift = paged ? __builtin_ctz((unsigned)a.g.page_size) : 0;
    p.q = (const unsigned char*)a.q; p.k = (const unsigned char*)a.k; p.v = (const unsigned char*)a.v; p.out = (unsigned char*)a.out;
    p.qs = bytes(a.qs); p.ks = bytes(a.ks); p.vs = bytes(a.vs); p.os = bytes(a.os);
    p.row_off = a.row_off; p.table = a.table; p.lens = a.lens; p.scale = a.scale; p.lse = a.lse;
    if (s.dtype == PKV_BF16) {
        if (few_rows(s, a.max_rows)) return s.D == 128 ? launch_stream<128>(s, p, a.ws, st) : launch_stream<64>(s, p, a.ws, st);
        if (paged) return s.D == 128 ? launch_tiles<128, true>(s, p, a.ws, st) : launch_tiles<64, true>(s, p, a.ws, st);
        return s.D == 128 ? launch_tiles<128, false>(s, p, a.ws, st) : launch_tiles<64, false>(s, p, a.ws, st);
    }
    const dim3 grid((unsigned)s.T, (unsigned)s.H, (unsigned)s.L);
    if (s.D == 128) hipLaunchKernelGGL(attn_rows_kernel<128>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(attn_rows_kernel<64>, grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace pkv
