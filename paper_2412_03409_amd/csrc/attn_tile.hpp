// What the kernels of attention of packed rows have in common: the softmax state of 32 rows and the two products on the matrix cores,
// copies into shared memory, joining parts.
#pragma once

#include "packed.hpp"
#include "fast_div.hpp"
#include "packed_rules.hpp"

namespace pkv {

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

// ---- bf16: the matrix cores ----------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef unsigned short v2u16_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v4i16_t lds_v4i16_t;

constexpr int kTileRows = 128;      // rows of a workgroup
constexpr int kStage = 64;          // keys that a workgroup stages at a time
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
    // in all, for twice the second products, which a stream of keys that HBM bounds hides.  CHECK: values that are infinite or NaN are kept
    // from rows that do not see them.
    template <int NKT, bool MASKED, bool SPLIT = false, bool CHECK = MASKED>
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
                    if constexpr (CHECK) { s[kt][8 * sl + e] = p0; s[kt][8 * sl + e + 1] = p1; }
                }
                pf[sl] = __builtin_bit_cast(bf16x8_t, make_uint4(pk[0], pk[1], pk[2], pk[3]));
                if constexpr (SPLIT) rest[sl] = __builtin_bit_cast(bf16x8_t, make_uint4(rk[0], rk[1], rk[2], rk[3]));
            }
            sum += psum;
            if constexpr (CHECK) {
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

// How many states all of some rows see, and how many some of them do
struct Limits { int all, some; };

}  // namespace pkv
