// Causal attention of packed rows: whole prompts of different lengths over their own packed keys, and chunks of new rows over a
// paged cache.  Both are one operator with two places to read keys from: row i of a sequence's n rows sees the keys
// 0 ... len - n + i, where len = n for a prompt.  Query heads that share a KV head are rows of one tile, row = token * heads + head:
// the keys are read once for all of them, and a tile's diagonal is as narrow as its tokens are few.
//
//  attn_tiles_kernel  bf16, many rows.  A workgroup has 128 rows of one (sequence, KV head), a wavefront 32 of them.  Keys and
//                     values stream through LDS 64 at a time (asynchronous copies, two buffer pairs).  Bound: the matrix cores
//                     and the softmax next to them.
//  attn_stream_kernel bf16, at most 32 rows per (sequence, KV head): decode steps.  A wavefront streams 32 keys at a time through
//                     LDS of its own.  All keys of a launch are one sequence of blocks that the wavefronts share out evenly,
//                     wherever the units begin and end.  Bound: HBM.
//  attn_merge_*       join the parts of a tile or unit that several workgroups or wavefronts worked on.
//  attn_rows_kernel   fp32: a wavefront per (row, head, layer).  The keys stream past one row: LPR lanes hold a key
//                     row, scores meet by shuffles, softmax online (running maximum and sum, everything fp32).
//
// The two bf16 kernels work as the prompt attention of rectangular batches does: S^T[32 keys x 32 rows] = K Q^T and
// O^T[32 columns x 32 rows] += V^T P^T with v_mfma_f32_32x32x16_bf16.  A lane holds one row's scores, so the softmax state is a
// scalar per lane, and the probabilities, rounded to bf16 against the running maximum, are the second product's operand where
// they are.  V^T comes from row-major V by the transposing LDS read.
#include "pkv_common.hpp"
#include "fast_div.hpp"

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
    const int t = blockIdx.x, h = blockIdx.y * 4 + wv, l = blockIdx.z;
    if (h >= p.H) return;
    // the sequence of row t: how many end at t or before it
    int s = 0;
    for (int i = lane; i < p.S; i += kWave) s += p.row_off[i + 1] <= t;
    s = wave_sum(s);
    if (s >= p.S) return;
    const int first = p.row_off[s], n = p.row_off[s + 1] - first, i = t - first;
    if (first < 0 || i < 0 || i >= p.max_rows) return;
    const int count = i + 1 + entries(p, s, l) - n;             // keys that the row sees
    const int32_t* pages = p.table + ((int64_t)s * p.layers + p.l0 + l) * p.max_pages;
    const int g = h / p.grp;
    const float4 q = *(const float4*)(p.q + p.qs.l * l + p.qs.h * h + p.qs.n * t + sub * 16);
    const float scale = p.scale[l] * kLog2e;
    float m = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto weigh = [](float4& x, float c) { x.x *= c; x.y *= c; x.z *= c; x.w *= c; };
    for (int j0 = 0; j0 < count; j0 += RG * U) {
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
            sc[u] = real[u] ? d * scale : -INFINITY;
            mx = fmaxf(mx, sc[u]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx, corr = __builtin_amdgcn_exp2f(m - ref);
        m = mx;
        sum *= corr;
        weigh(o, corr);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = __builtin_amdgcn_exp2f(sc[u] - ref);
            sum += w;
            o.x = fmaf(w, vr[u].x, o.x); o.y = fmaf(w, vr[u].y, o.y); o.z = fmaf(w, vr[u].z, o.z); o.w = fmaf(w, vr[u].w, o.w);
        }
    }
    // the row groups hold every RG-th key each
    float all = m;
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) all = fmaxf(all, __shfl_xor(all, x, kWave));
    const float ref = all == -INFINITY ? 0.f : all, corr = __builtin_amdgcn_exp2f(m - ref);
    sum *= corr;
    weigh(o, corr);
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) {
        sum += __shfl_xor(sum, x, kWave);
        o.x += __shfl_xor(o.x, x, kWave); o.y += __shfl_xor(o.y, x, kWave);
        o.z += __shfl_xor(o.z, x, kWave); o.w += __shfl_xor(o.w, x, kWave);
    }
    if (rg != 0) return;
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

__device__ __forceinline__ void copy_to_lds(const unsigned char* src, unsigned char* dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
}

// Softmax state and output of the 32 rows of a wavefront: row lane % 32; register r of o[dt] is column
// 32 dt + 8 (r / 4) + 4 (lane / 32) + r % 4.
template <int D>
struct RowTile {
    bf16x8_t q[D / 16];
    f32x16_t o[D / 32];
    float m, sum;             // running maximum of score * qs, and this half's part of the sum
    uint32_t koff[D / 16], voff[D / 32][2];   // byte offsets of the lane's fragment reads in a staged 32-key tile

    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        sum = 0.f;
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
    // 16x ... 16x+15, and tiles from `tiles` on are seen by no row of the wavefront.  Each tile has its own reference, the maximum up
    // to its end: the probabilities are rounded against it.
    template <int NKT, bool MASKED>
    __device__ __forceinline__ void attend(const unsigned char* sK, const unsigned char* sV, float qs, int lane, int lim, uint32_t bad,
                                           int tiles) {
        constexpr int ROWB = D * 2, NJ = D / 16, NDT = D / 32, CPR = D / 8;
        const int hf = lane >> 5;
        f32x16_t s[NKT];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *(const uint4*)(sK + kt * 32 * ROWB + koff[j]));
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[j], s[kt], 0, 0, 0);
            }
        }
        if constexpr (MASKED) {
            const int mine = lim - 4 * hf;                    // register r holds key 8 (r/4) + r%4 + 4 hf
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool see = 32 * kt + 8 * (r >> 2) + (r & 3) <= mine && !((bad >> (2 * kt + (r >> 3))) & 1u);
                    s[kt][r] = see ? s[kt][r] : -INFINITY;
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
        float mref[NKT], corr[NKT], top = mx[0];
        bool later = false;                                  // the second tile moves the maximum
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) { mref[kt] = m; corr[kt] = 1.f; top = fmaxf(top, mx[kt]); }
        // most stages of a long prompt move no row's maximum: one look, before the two halves of a row exchange theirs
        if (__builtin_amdgcn_ballot_w64(top * qs > m)) {
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) {
                const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx[kt]), __float_as_uint(mx[kt]), false, false);
                mref[kt] = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * qs);
                corr[kt] = mref[kt] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mref[kt]);
                if (kt == 1) later = __builtin_amdgcn_ballot_w64(mref[kt] > m) != 0;
                m = mref[kt];
            }
            if (__builtin_amdgcn_ballot_w64(corr[0] != 1.f)) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] *= corr[0];
            }
        }
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
            if (MASKED && kt >= tiles) break;
            const float ref = mref[kt] == -INFINITY ? 0.f : mref[kt];      // no score so far
            bf16x8_t pf[2];
            float psum = 0.f;
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
                uint32_t pk[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kt][8 * sl + e], qs, -ref));
                    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kt][8 * sl + e + 1], qs, -ref));
                    psum += p0 + p1;
                    pk[e / 2] = pack_bf16(p0, p1);
                    if constexpr (MASKED) { s[kt][8 * sl + e] = p0; s[kt][8 * sl + e + 1] = p1; }
                }
                pf[sl] = __builtin_bit_cast(bf16x8_t, make_uint4(pk[0], pk[1], pk[2], pk[3]));
            }
            sum = fmaf(sum, corr[kt], psum);
            if (kt == 1 && later) {
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[dt][r] *= corr[kt];
            }
            if constexpr (MASKED) {
                // An infinite or NaN value that some rows must not see would reach them as 0 * value: such a tile is added up row by
                // row, over the keys that each of them sees.  (The look costs a masked stage 2 NDT x 8 packed maxima.)
                v2u16_t big = {0, 0};
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const uint2 w = __builtin_bit_cast(uint2, lds_read_tr(sV + (32 * kt + 16 * x) * ROWB + voff[dt][y]));
                            big = __builtin_elementwise_max(big, __builtin_bit_cast(v2u16_t, w.x & 0x7fff7fffu));
                            big = __builtin_elementwise_max(big, __builtin_bit_cast(v2u16_t, w.y & 0x7fff7fffu));
                        }
                if (__builtin_amdgcn_ballot_w64(big.x >= 0x7f80 || big.y >= 0x7f80)) {
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
            for (int sl = 0; sl < 2; ++sl)
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) {
                    const unsigned char* sVs = sV + (32 * kt + 16 * sl) * ROWB;
                    const v4i16_t a0 = lds_read_tr(sVs + voff[dt][0]), a1 = lds_read_tr(sVs + voff[dt][1]);
                    const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[sl], o[dt], 0, 0, 0);
                }
        }
    }

    // the whole row sum, in both halves
    __device__ __forceinline__ float total() const { return sum + __shfl_xor(sum, 32, kWave); }

    // the finished row (16 bytes per lane and 8 columns: the halves of a row swap their pieces)
    __device__ __forceinline__ void store(unsigned char* row, int hf, float inv, bool real) const {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int g = 0; g < 4; g += 2) {
                uint32_t w[2][2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    w[x][0] = pack_bf16(o[dt][4 * (g + x)] * inv, o[dt][4 * (g + x) + 1] * inv);
                    w[x][1] = pack_bf16(o[dt][4 * (g + x) + 2] * inv, o[dt][4 * (g + x) + 3] * inv);
                }
                const auto s0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                if (real) *(uint4*)(row + 2 * (32 * dt + 8 * (g + hf))) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
            }
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

// scale in units of log2, above 0 so that a masked -inf stays one (NaN stays NaN)
__device__ __forceinline__ float score_scale(float sc) {
    const float a = fabsf(sc) * kLog2e;
    return a < 1e-30f ? 1e-30f : a;
}

struct Sequence { int first, n, rows; };    // first packed row, rows, rows of this call (times the heads of a KV head)

// What a row of a tile or unit is: row = token * grp + head of the KV head
struct RowAt { int token, head; };
__device__ __forceinline__ RowAt row_at(int row, FastDiv grp) {
    const DivMod x = div_mod(row, grp);
    return {x.q, x.r};
}

struct TileParams {
    PackedParams a;
    FastDiv grp, by_heads, by_hkv, by_tail, by_tiles, by_parts;
    int heads, tiles, parts;       // L * Hkv; tiles of all sequences at most; parts of a tile's keys at most
    int heads_per_xcd;             // 0: the heads do not divide up
    float* part_o;                 // [heads][tiles][parts][128][D]
    float2* part_ms;
};
constexpr int kPartStages = 6;     // stages of a part at least

// Tile tt: sequence by sequence, the last tile of a sequence first (its rows see the most).  false: there are fewer.
__device__ __forceinline__ bool find_tile(const PackedParams& p, int grp, int tt, int lane, Sequence& sq, int& s, int& tile) {
    int base = 0;
    for (int c = 0; c < p.S; c += kWave) {
        const int i = c + lane;
        int first = 0, n = 0;
        if (i < p.S) {
            const int last = p.row_off[i + 1];
            first = p.row_off[i];
            n = first >= 0 && last <= p.T ? max(0, last - first) : 0;
        }
        const int rows = (p.max_rows > 0 ? min(n, p.max_rows) : n) * grp, tiles = (rows + kTileRows - 1) / kTileRows;
        int incl = tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int up = __shfl_up(incl, d, kWave);
            if (lane >= d) incl += up;
        }
        const unsigned long long at = __builtin_amdgcn_ballot_w64(base + incl > tt);
        if (at != 0) {
            const int j = __builtin_ctzll(at);
            s = c + j;
            sq = {__builtin_amdgcn_readlane(first, j), __builtin_amdgcn_readlane(n, j), __builtin_amdgcn_readlane(rows, j)};
            tile = base + __builtin_amdgcn_readlane(incl, j) - 1 - tt;
            return true;
        }
        base += __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    return false;
}

template <bool PAGED>
struct TileKeys { int len, before, end, nst, parts; };   // keys; keys in front of the first new row; keys that the tile sees; stages; parts

template <bool PAGED>
__device__ __forceinline__ TileKeys<PAGED> tile_keys(const TileParams& p, const Sequence& sq, int s, int l, int tile) {
    TileKeys<PAGED> k;
    k.len = PAGED ? entries(p.a, s, l) : sq.n;
    k.before = k.len - sq.n;                                    // below 0: the first rows see nothing
    const int last = __builtin_amdgcn_readfirstlane(row_at(min(sq.rows, (tile + 1) * kTileRows) - 1, p.grp).token);
    k.end = max(0, min(k.len, k.before + last + 1));
    k.nst = (k.end + kStage - 1) / kStage;
    k.parts = max(1, min(p.parts, k.nst / kPartStages));
    return k;
}

struct TileAt { int head, tt, part; };
// Which tile a workgroup has.  With heads in eighths every head stays on one XCD: the tiles of a head run next to each other and
// share its keys through that XCD's L2; the last heads of an XCD are taken together, so that the launch does not end on the long
// tiles of a single one.  Else, and where tiles come in parts, heads alternate and the tiles go from long to short.
__device__ __forceinline__ TileAt tile_at(const TileParams& p, int bid) {
    if (p.parts == 1 && p.heads_per_xcd > 0) {
        const int xcd = bid % kXcds, j = bid / kXcds, lead = p.heads_per_xcd - (int)p.by_tail.d;
        if (j < lead * p.tiles) {
            const DivMod x = uniform_div_mod(j, p.by_tiles);
            return {xcd * p.heads_per_xcd + x.q, x.r, 0};
        }
        const DivMod x = uniform_div_mod(j - lead * p.tiles, p.by_tail);
        return {xcd * p.heads_per_xcd + lead + x.r, x.q, 0};
    }
    const DivMod x = uniform_div_mod(bid, p.by_heads), y = uniform_div_mod(x.q, p.by_parts);
    return {x.r, y.q, y.r};
}

template <int D, bool PAGED>
__global__ void __launch_bounds__(256, 2)
attn_tiles_kernel(TileParams p) {
    constexpr int ROWB = D * 2, CPR = D / 8, kInst = kStage * ROWB / 1024 / 4;    // copies per wavefront, stage and tensor: 16 rows
    __shared__ __attribute__((aligned(1024))) unsigned char sKa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVa[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sKb[kStage * ROWB];
    __shared__ __attribute__((aligned(1024))) unsigned char sVb[kStage * ROWB];
    const PackedParams& a = p.a;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const TileAt at = tile_at(p, (int)blockIdx.x);
    Sequence sq;
    int s, tile;
    if (!find_tile(a, a.grp, at.tt, lane, sq, s, tile)) return;
    const DivMod lh = uniform_div_mod(at.head, p.by_hkv);
    const int l = lh.q, g = lh.r;
    const TileKeys<PAGED> keys = tile_keys<PAGED>(p, sq, s, l, tile);
    if (at.part >= keys.parts) return;
    const int st0 = keys.nst * at.part / keys.parts, st1 = keys.nst * (at.part + 1) / keys.parts;

    // this wavefront's rows
    const int r0 = tile * kTileRows + wv * 32, ln = lane & 31, hf = lane >> 5, row = r0 + ln;
    const bool mine = r0 < sq.rows, real = row < sq.rows;
    const RowAt ra = row_at(real ? row : mine ? r0 : 0, p.grp);               // (rows that do not exist repeat one that does)
    const int lim = keys.before + ra.token;                                   // the last key that the row sees
    const int lim_first = keys.before + __builtin_amdgcn_readfirstlane(row_at(mine ? r0 : 0, p.grp).token);
    const int lim_last = keys.before + __builtin_amdgcn_readfirstlane(row_at(min(sq.rows, r0 + 32) - 1, p.grp).token);
    const int h = g * a.grp + ra.head;
    const int64_t t = sq.first + ra.token;

    // Keys and values of a stage: a wavefront copies 16 rows of each, which lie in one page.
    const unsigned char *kb, *vb;
    const int32_t* pages = nullptr;
    if constexpr (PAGED) {
        pages = a.table + ((int64_t)s * a.layers + a.l0 + l) * a.max_pages;
        kb = a.k; vb = a.v;
    } else {
        kb = a.k + a.ks.l * l + a.ks.h * g + a.ks.n * sq.first;
        vb = a.v + a.vs.l * l + a.vs.h * g + a.vs.n * sq.first;
    }
    int cp_row[kInst], cp_col[kInst];
#pragma unroll
    for (int i = 0; i < kInst; ++i) {
        const int idx = (wv * kInst + i) * 64 + lane, r = idx / CPR;
        cp_row[i] = r;
        cp_col[i] = 16 * ((idx % CPR) ^ swz<CPR>(r));
    }
    // Page ids ahead of their use: lane i has that of the i-th group of 16 keys from ids0 on, `next` the 64 groups behind them.
    int ids = 0, next = 0, ids0 = st0 * 4;
    unsigned long long bad_now = 0, bad_next = 0;
    auto load_ids = [&](int group) {
        const int key = min((group + lane) * 16, max(keys.end - 1, 0));
        return keys.end > 0 ? pages[key >> a.shift] : 0;
    };
    auto check_ids = [&](int& x) {
        const bool out = (uint32_t)x >= (uint32_t)a.num_pages;
        if (out) x = 0;
        return __builtin_amdgcn_ballot_w64(out);
    };
    if constexpr (PAGED) {
        ids = load_ids(ids0);
        next = load_ids(ids0 + kWave);
        bad_now = check_ids(ids);
        bad_next = check_ids(next);
    }
    auto bad_of = [&](int st) -> uint32_t {
        if constexpr (!PAGED) return 0u;
        const int x = st * 4 - ids0;      // a stage behind: its groups may have moved out at the front
        return x < 0 ? 0u : (uint32_t)((bad_now >> x) & 15u);
    };
    auto issue = [&](int st, unsigned char* dK, unsigned char* dV) -> uint32_t {
        uint32_t bad = 0;
        if constexpr (PAGED) {
            if (st * 4 >= ids0 + kWave) {
                ids = next; bad_now = bad_next; ids0 += kWave;
                next = load_ids(ids0 + kWave);
                bad_next = check_ids(next);
            }
            bad = bad_of(st);
            const int64_t id = __builtin_amdgcn_readlane(ids, st * 4 + wv - ids0);
            const int64_t base = ((id * a.Hkv + g) << a.shift) * ROWB;
#pragma unroll
            for (int i = 0; i < kInst; ++i) {
                const int key = min(st * kStage + cp_row[i], keys.end - 1);
                const uint32_t off = (uint32_t)((key & ((1 << a.shift) - 1)) * ROWB + cp_col[i]);
                copy_to_lds(kb + base + off, dK + (wv * kInst + i) * 1024);
                copy_to_lds(vb + base + off, dV + (wv * kInst + i) * 1024);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kInst; ++i) {
                const int64_t key = min(st * kStage + cp_row[i], keys.end - 1);
                copy_to_lds(kb + a.ks.n * key + cp_col[i], dK + (wv * kInst + i) * 1024);
                copy_to_lds(vb + a.vs.n * key + cp_col[i], dV + (wv * kInst + i) * 1024);
            }
        }
        return bad;
    };
    uint32_t bad_a = 0, bad_b = 0;
    if (st0 < st1) bad_a = issue(st0, sKa, sVa);

    const float sc = a.scale[l], qs = score_scale(sc);
    RowTile<D> tl;
    tl.load_q(a.q + a.qs.l * l + a.qs.h * h + a.qs.n * t, hf, sc < 0.f);
    tl.clear();
    tl.offsets(lane);

    auto sync = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0F70);                  // vmcnt(0): this wavefront's part of the stage has landed
        __syncthreads();                                     // ... and everybody's; the other pair is free again
    };
    auto attend = [&](int st, const unsigned char* sK, const unsigned char* sV, uint32_t bad) {
        const int key0 = st * kStage;
        if (!mine) return;
        if (key0 + kStage - 1 <= lim_first && bad == 0) tl.template attend<2, false>(sK, sV, qs, lane, 0, 0u, 2);
        else if (key0 <= lim_last) tl.template attend<2, true>(sK, sV, qs, lane, lim - key0, bad, key0 + 32 <= lim_last ? 2 : 1);
    };
    for (int st = st0; st < st1; st += 2) {
        sync();
        if (st + 1 < st1) bad_b = issue(st + 1, sKb, sVb);
        attend(st, sKa, sVa, bad_a);
        if (st + 1 >= st1) break;
        sync();
        if (st + 2 < st1) bad_a = issue(st + 2, sKa, sVa);
        attend(st + 1, sKb, sVb, bad_b);
    }
    if (!mine) return;
    const float all = tl.total();
    if (keys.parts > 1) {
        const int64_t slot = (((int64_t)at.head * p.tiles + at.tt) * p.parts + at.part) * kTileRows + wv * 32 + ln;
        if (real) tl.store_part(p.part_o + slot * D, p.part_ms + slot, hf, all);
        return;
    }
    tl.store(a.out + a.os.l * l + a.os.h * h + a.os.n * t, hf, all == 0.f ? 0.f : 1.f / all, real);
    if (!PAGED && real && hf == 0)
        a.lse[(int64_t)a.L * a.H * sq.first + (int64_t)(l * a.H + h) * sq.n + ra.token] = kLn2 * (tl.m + __builtin_amdgcn_logf(all));
}

// Joins the parts of a tile's rows: a wavefront takes 4 columns per lane of 256 / D rows at a time.
template <int D, bool PAGED>
__global__ void __launch_bounds__(256)
attn_merge_tiles_kernel(TileParams p) {
    constexpr int LPR = D / 4, RPB = 256 / LPR;
    const PackedParams& a = p.a;
    const int lane = threadIdx.x & (kWave - 1);
    const DivMod x = uniform_div_mod((int)blockIdx.x, p.by_heads);
    Sequence sq;
    int s, tile;
    if (!find_tile(a, a.grp, x.q, lane, sq, s, tile)) return;
    const DivMod lh = uniform_div_mod(x.r, p.by_hkv);
    const TileKeys<PAGED> keys = tile_keys<PAGED>(p, sq, s, lh.q, tile);
    if (keys.parts == 1) return;
    const int in_tile = (int)blockIdx.y * RPB + threadIdx.x / LPR, row = tile * kTileRows + in_tile, c = 4 * (threadIdx.x % LPR);
    if (row >= sq.rows) return;
    const int64_t slot0 = ((int64_t)x.r * p.tiles + x.q) * p.parts * kTileRows + in_tile;
    float m = -INFINITY;
    for (int i = 0; i < keys.parts; ++i) m = fmaxf(m, p.part_ms[slot0 + i * kTileRows].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < keys.parts; ++i) {
        const int64_t slot = slot0 + i * kTileRows;
        const float2 ms = p.part_ms[slot];
        const float4 y = *(const float4*)(p.part_o + slot * D + c);
        const float w = __builtin_amdgcn_exp2f(ms.x - ref);
        sum = fmaf(w, ms.y, sum);
        o.x = fmaf(w, y.x, o.x); o.y = fmaf(w, y.y, o.y); o.z = fmaf(w, y.z, o.z); o.w = fmaf(w, y.w, o.w);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const RowAt ra = row_at(row, p.grp);
    const int h = lh.r * a.grp + ra.head;
    *(uint2*)(a.out + a.os.l * lh.q + a.os.h * h + a.os.n * (int64_t)(sq.first + ra.token) + 2 * c) =
        make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (!PAGED && c == 0)
        a.lse[(int64_t)a.L * a.H * sq.first + (int64_t)(lh.q * a.H + h) * sq.n + ra.token] = kLn2 * (m + __builtin_amdgcn_logf(sum));
}

// ---- few rows: the keys of a launch shared out evenly over the wavefronts ---------------------------------
struct StreamParams {
    PackedParams a;
    FastDiv grp, by_layers;         // by_layers: layers of the call
    int segs, waves;                // S * L
    int* share;                     // workspace: blocks of a wavefront
    int* start;                     // [segs]: first block of a segment (segments that have blocks)
    float* part_o;                  // [2 * waves][32][D]
    float2* part_ms;
};
constexpr int kLeastBlocks = 2;     // of a wavefront

struct Segment { int s, l, first, n, rows, len, end, blocks; };   // rows: of this call, times the heads; end: keys that some row sees

__device__ __forceinline__ Segment segment(const StreamParams& p, int i) {
    Segment x;
    const DivMod sl = div_mod(i, p.by_layers);
    x.s = sl.q; x.l = sl.r;
    const int last = p.a.row_off[x.s + 1];
    x.first = p.a.row_off[x.s];
    x.n = x.first >= 0 && last <= p.a.T ? max(0, last - x.first) : 0;
    x.len = entries(p.a, x.s, x.l);
    const int rows = min(x.n, p.a.max_rows);
    x.rows = rows * p.a.grp;
    x.end = x.n > 0 ? max(0, min(x.len, x.len - x.n + rows)) : 0;
    x.blocks = (x.end + kBlockKeys - 1) / kBlockKeys;
    return x;
}
__device__ __forceinline__ Segment uniform_segment(const StreamParams& p, int i) {
    Segment x = segment(p, i);
    x.s = __builtin_amdgcn_readfirstlane(x.s); x.l = __builtin_amdgcn_readfirstlane(x.l);
    x.first = __builtin_amdgcn_readfirstlane(x.first); x.n = __builtin_amdgcn_readfirstlane(x.n);
    x.rows = __builtin_amdgcn_readfirstlane(x.rows); x.len = __builtin_amdgcn_readfirstlane(x.len);
    x.end = __builtin_amdgcn_readfirstlane(x.end); x.blocks = __builtin_amdgcn_readfirstlane(x.blocks);
    return x;
}

template <int D>
__global__ void __launch_bounds__(128, 128 / D)
attn_stream_kernel(StreamParams p) {
    constexpr int ROWB = D * 2, CPR = D / 8, kBytes = kBlockKeys * ROWB, kInst = 16 * ROWB / 1024;   // copies per 16 keys and tensor
    __shared__ __attribute__((aligned(1024))) unsigned char sKa[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sVa[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sKb[2][kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char sVb[2][kBytes];
    const PackedParams& a = p.a;
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 2 + wv), ln = lane & 31, hf = lane >> 5;

    // the launch's blocks, and this wavefront's: segment by segment, KV head by KV head
    int sum = 0;
    for (int i = lane; i < p.segs; i += kWave) sum += segment(p, i).blocks;
    const int all_blocks = __builtin_amdgcn_readfirstlane(wave_sum(sum)) * a.Hkv;
    const int share = max(kLeastBlocks, (all_blocks + p.waves - 1) / p.waves);
    if (wave == 0 && lane == 0) *p.share = share;
    const int b0 = (int)min((int64_t)wave * share, (int64_t)all_blocks), b1 = (int)min((int64_t)b0 + share, (int64_t)all_blocks);
    if (b0 >= b1) return;
    int seg = 0, before = 0;                                   // segment of block b0, blocks in front of it
    for (int c = 0; c < p.segs; c += kWave) {
        const int mine = c + lane < p.segs ? segment(p, c + lane).blocks : 0;
        int incl = mine;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int up = __shfl_up(incl, d, kWave);
            if (lane >= d) incl += up;
        }
        const unsigned long long at = __builtin_amdgcn_ballot_w64((before + incl) * a.Hkv > b0);
        if (at != 0) {
            const int j = __builtin_ctzll(at);
            seg = c + j;
            before += __builtin_amdgcn_readlane(incl, j) - __builtin_amdgcn_readlane(mine, j);
            break;
        }
        before += __builtin_amdgcn_readlane(incl, kWave - 1);
    }

    // where copies are asked for (`in`), and where the work is (`sg`): both walk the same blocks
    struct Cursor { int seg, g, blk; };
    Segment sg = uniform_segment(p, seg), in = sg;
    Cursor cw = {seg, 0, b0 - before * a.Hkv};
    cw.g = cw.blk / sg.blocks;
    cw.blk -= cw.g * sg.blocks;
    int seg_start = before * a.Hkv;                             // first block of the segment worked on
    Cursor ci = cw;
    auto step = [&](Cursor& c, Segment& x) -> bool {            // true: another segment
        if (++c.blk < x.blocks) return false;
        c.blk = 0;
        if (++c.g < a.Hkv) return false;
        c.g = 0;
        do { ++c.seg; x = uniform_segment(p, c.seg); } while (x.blocks == 0);    // (a block is left, so a segment is)
        return true;
    };
    int cp_row[kInst], cp_col[kInst];                           // of 16 keys
#pragma unroll
    for (int i = 0; i < kInst; ++i) {
        const int idx = i * 64 + lane, r = idx / CPR;
        cp_row[i] = r;
        cp_col[i] = idx % CPR;
    }
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
            const int64_t base = ((id * a.Hkv + ci.g) << a.shift) * ROWB;
#pragma unroll
            for (int i = 0; i < kInst; ++i) {
                const int r = 16 * x + cp_row[i];
                const int key = min(ci.blk * kBlockKeys + r, in.end - 1);
                const uint32_t off = (uint32_t)((key & ((1 << a.shift) - 1)) * ROWB + 16 * (cp_col[i] ^ swz<CPR>(r)));
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
        lim = sg.len - sg.n + ra.token;
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
        if (key0 + kBlockKeys - 1 <= sg.len - sg.n && bad == 0) tl.template attend<1, false>(sK, sV, qs, lane, 0, 0u, 1);
        else tl.template attend<1, true>(sK, sV, qs, lane, lim - key0, bad, 1);
    };
    // one block of the work: `more` blocks are in flight behind it
    auto work = [&](int b, const unsigned char* sK, const unsigned char* sV, uint32_t bad) {
        attend(sK, sV, bad);
        const bool whole = cw.blk + 1 == sg.blocks;
        if (whole || b + 1 == b1) {
            end(whole);
            if (b + 1 < b1) {
                const int old = sg.blocks;
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

// Joins the pieces of a unit's row; rows of units without a block get zeros.  One workgroup per (unit, row): D / 4 lanes per
// piece, the pieces dealt out over the groups of lanes.
template <int D>
__global__ void __launch_bounds__(256)
attn_merge_stream_kernel(StreamParams p) {
    constexpr int LPP = D / 4, PG = 256 / LPP;
    __shared__ float s_m[PG], s_sum[PG];
    __shared__ float4 s_o[PG][LPP];
    const PackedParams& a = p.a;
    const int i = (int)blockIdx.x / a.Hkv, g = (int)blockIdx.x % a.Hkv, row = (int)blockIdx.y;
    const Segment x = uniform_segment(p, i);
    if (row >= x.rows) return;
    const RowAt ra = row_at(row, p.grp);
    const int c = threadIdx.x % LPP, pg = threadIdx.x / LPP, h = g * a.grp + ra.head;
    unsigned char* out = a.out + a.os.l * x.l + a.os.h * h + a.os.n * (int64_t)(x.first + ra.token) + 8 * c;
    if (x.blocks == 0) {
        if (pg == 0) *(uint2*)out = make_uint2(0u, 0u);
        return;
    }
    const int share = *p.share, u0 = p.start[i] + g * x.blocks, w0 = u0 / share, w1 = (u0 + x.blocks - 1) / share;
    if (w0 == w1) return;                                       // one wavefront has written it
    float m = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // a running maximum, so that every piece is read once
    for (int w = w0 + pg; w <= w1; w += PG) {
        const int64_t slot = (int64_t)(2 * w + (w == w0 ? 1 : 0)) * kFewRows + row;
        const float2 ms = p.part_ms[slot];
        const float4 y = *(const float4*)(p.part_o + slot * D + 4 * c);
        const float mx = fmaxf(m, ms.x), ref = mx == -INFINITY ? 0.f : mx;
        const float c0 = __builtin_amdgcn_exp2f(m - ref), c1 = __builtin_amdgcn_exp2f(ms.x - ref);
        sum = fmaf(sum, c0, ms.y * c1);
        o.x = fmaf(o.x, c0, y.x * c1); o.y = fmaf(o.y, c0, y.y * c1); o.z = fmaf(o.z, c0, y.z * c1); o.w = fmaf(o.w, c0, y.w * c1);
        m = mx;
    }
    if (c == 0) { s_m[pg] = m; s_sum[pg] = sum; }
    s_o[pg][c] = o;
    __syncthreads();
    if (pg != 0) return;
    float all = -INFINITY;
#pragma unroll
    for (int k = 0; k < PG; ++k) all = fmaxf(all, s_m[k]);
    const float ref = all == -INFINITY ? 0.f : all;
    sum = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < PG; ++k) {
        const float w = __builtin_amdgcn_exp2f(s_m[k] - ref);
        const float4 y = s_o[k][c];
        sum = fmaf(w, s_sum[k], sum);
        o.x = fmaf(w, y.x, o.x); o.y = fmaf(w, y.y, o.y); o.z = fmaf(w, y.z, o.z); o.w = fmaf(w, y.w, o.w);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    *(uint2*)out = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

// ---- launches ------------------------------------------------------------------------------------------
constexpr int kStreamWorkgroups = 2;          // of a compute unit: 64 KB of LDS each at D = 128
constexpr int kTileSlots = 2;                 // workgroups of attn_tiles_kernel that a compute unit holds
constexpr int kTailTiles = 256;               // workgroups of an XCD at the end of a launch whose heads are taken together

static bool few_rows(const pkv_packed& s, int max_rows) { return max_rows > 0 && (int64_t)max_rows * (s.H / s.Hkv) <= kFewRows; }
static int stream_waves(const pkv_packed& s) { return compute_units() * kStreamWorkgroups * 2 * (128 / s.D); }

// tiles of all sequences at most, and the parts that a tile's keys are split into so that the launch fills the chip once
struct TileCount { long long tiles, heads; int parts; };
static TileCount tile_count(const pkv_packed& s) {
    TileCount c;
    const long long grp = s.H / s.Hkv;
    c.heads = (long long)s.L * s.Hkv;
    c.tiles = ((long long)s.T * grp) / kTileRows + (s.S < s.T ? s.S : s.T);
    const long long slots = (long long)compute_units() * kTileSlots, items = c.tiles * c.heads;
    c.parts = (int)(items >= slots ? 1 : slots / items < 16 ? slots / items : 16);
    return c;
}

// grids and block numbers are 32 bits wide
bool packed_attn_fits(const pkv_packed& s, const pkv_paging* g) {
    const TileCount c = tile_count(s);
    if (c.tiles * c.heads * c.parts > 0x7fffffffll) return false;
    return !g || (double)s.S * s.L * s.Hkv * g->max_pages * g->page_size / kBlockKeys < 2147483648.0;
}

size_t packed_attn_ws_bytes(const pkv_packed& s, int max_rows) {
    if (s.dtype != PKV_BF16) return 0;
    if (few_rows(s, max_rows)) {
        const size_t slots = (size_t)2 * stream_waves(s) * kFewRows;
        return 256 + ((size_t)s.S * s.L * 4 + 255) / 256 * 256 + slots * (sizeof(float2) + s.D * sizeof(float));
    }
    const TileCount c = tile_count(s);
    return c.parts == 1 ? 0 : (size_t)(c.tiles * c.heads * c.parts) * kTileRows * (sizeof(float2) + s.D * sizeof(float));
}

template <int D, bool PAGED>
static hipError_t launch_tiles(const pkv_packed& s, const PackedParams& a, void* ws, hipStream_t st) {
    const TileCount c = tile_count(s);
    const long long items = c.tiles * c.heads;
    TileParams p;
    p.a = a;
    p.heads = (int)c.heads; p.tiles = (int)c.tiles; p.parts = c.parts;
    p.heads_per_xcd = c.heads % kXcds == 0 ? (int)(c.heads / kXcds) : 0;
    const long long tail = (kTailTiles + c.tiles - 1) / c.tiles;
    p.grp = fast_div(a.grp); p.by_heads = fast_div(c.heads); p.by_hkv = fast_div(s.Hkv); p.by_tiles = fast_div(c.tiles);
    p.by_tail = fast_div(p.heads_per_xcd > 0 && tail < p.heads_per_xcd ? tail : p.heads_per_xcd > 0 ? p.heads_per_xcd : 1);
    p.by_parts = fast_div(c.parts);
    p.part_o = (float*)ws;
    p.part_ms = (float2*)(p.part_o + (size_t)(items * c.parts) * kTileRows * D);
    hipLaunchKernelGGL((attn_tiles_kernel<D, PAGED>), dim3((unsigned)(items * c.parts)), dim3(256), 0, st, p);
    if (c.parts > 1)
        hipLaunchKernelGGL((attn_merge_tiles_kernel<D, PAGED>), dim3((unsigned)items, kTileRows * (D / 4) / 256), dim3(256), 0, st, p);
    return hipGetLastError();
}

template <int D>
static hipError_t launch_stream(const pkv_packed& s, const PackedParams& a, void* ws, hipStream_t st) {
    StreamParams p;
    p.a = a;
    p.grp = fast_div(a.grp); p.by_layers = fast_div(s.L);
    p.segs = s.S * s.L; p.waves = stream_waves(s);
    p.share = (int*)ws;
    p.start = (int*)((char*)ws + 256);
    p.part_o = (float*)((char*)ws + 256 + ((size_t)p.segs * 4 + 255) / 256 * 256);
    p.part_ms = (float2*)(p.part_o + (size_t)2 * p.waves * kFewRows * D);
    hipLaunchKernelGGL(attn_stream_kernel<D>, dim3((unsigned)(p.waves / 2)), dim3(128), 0, st, p);
    hipLaunchKernelGGL(attn_merge_stream_kernel<D>, dim3((unsigned)(p.segs * s.Hkv), (unsigned)(a.max_rows * a.grp)), dim3(256), 0, st, p);
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
    const dim3 grid((unsigned)s.T, (unsigned)((s.H + 3) / 4), (unsigned)s.L);
    if (s.D == 128) hipLaunchKernelGGL(attn_rows_kernel<128>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(attn_rows_kernel<64>, grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace pkv
