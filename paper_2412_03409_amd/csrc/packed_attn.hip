// Causal attention of packed rows: whole prompts of different lengths over their own packed keys, and chunks of new rows over a
// paged cache.  Both are one operator with two places to read keys from: row i of a sequence's n rows sees the keys
// 0 ... len - n + i, where len = n for a prompt.
//
//  attn_rows_kernel   a wavefront per (row, head, layer); fp32 storage.  The keys stream past one row: LPR lanes hold a key
//                     row, scores meet by shuffles, softmax online (running maximum and sum, everything fp32).
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

template <bool BF16>
__device__ __forceinline__ void row_piece(const uint4& r, float* f) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        if constexpr (BF16) { f[2 * x] = __uint_as_float(w[x] << 16); f[2 * x + 1] = __uint_as_float(w[x] & 0xffff0000u); }
        else f[x] = __uint_as_float(w[x]);
    }
}

template <bool BF16, int D, bool PAGED>
__global__ void __launch_bounds__(256)
attn_rows_kernel(PackedParams p) {
    constexpr int VE = BF16 ? 8 : 4, LPR = D / VE, RG = kWave / LPR, U = 4;
    constexpr int kRow = D * (BF16 ? 2 : 4);
    const int lane = threadIdx.x & (kWave - 1), wv = threadIdx.x / kWave, sub = lane % LPR, rg = lane / LPR;
    const int t = blockIdx.x, h = blockIdx.y * 4 + wv, l = blockIdx.z;
    if (h >= p.H) return;
    // the sequence of row t: how many end at t or before it
    int s = 0;
    for (int i = lane; i < p.S; i += kWave) s += p.row_off[i + 1] <= t;
    s = wave_sum(s);
    if (s >= p.S) return;
    const int first = p.row_off[s], n = p.row_off[s + 1] - first, i = t - first;
    if (first < 0 || i < 0 || (PAGED && i >= p.max_rows)) return;
    int count = i + 1;
    const int32_t* pages = nullptr;
    const int g = h / p.grp;
    const unsigned char *kb, *vb;
    if constexpr (PAGED) {
        const int64_t seg = (int64_t)s * p.layers + p.l0 + l;
        count += min(p.lens[seg], p.max_pages << p.shift) - n;
        pages = p.table + seg * p.max_pages;
        kb = p.k; vb = p.v;
    } else {
        kb = p.k + p.ks.l * l + p.ks.h * g + p.ks.n * first;
        vb = p.v + p.vs.l * l + p.vs.h * g + p.vs.n * first;
    }
    float q[VE], o[VE];
    row_piece<BF16>(*(const uint4*)(p.q + p.qs.l * l + p.qs.h * h + p.qs.n * t + sub * 16), q);
    const float scale = p.scale[l] * kLog2e;
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] = 0.f;
    for (int j0 = 0; j0 < count; j0 += RG * U) {
        uint4 kr[U], vr[U];
        bool real[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * RG + rg;
            real[u] = j < count;
            kr[u] = vr[u] = make_uint4(0, 0, 0, 0);
            int64_t ka = 0, va = 0;
            if constexpr (PAGED) {
                const int id = real[u] ? pages[j >> p.shift] : -1;
                real[u] = (uint32_t)id < (uint32_t)p.num_pages;
                ka = va = ((((int64_t)id * p.Hkv + g) << p.shift) + (j & ((1 << p.shift) - 1))) * kRow;
            } else {
                ka = p.ks.n * j; va = p.vs.n * j;
            }
            if (real[u]) { kr[u] = *(const uint4*)(kb + ka + sub * 16); vr[u] = *(const uint4*)(vb + va + sub * 16); }
        }
        float sc[U], mx = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[VE], d = 0.f;
            row_piece<BF16>(kr[u], f);
#pragma unroll
            for (int e = 0; e < VE; ++e) d = fmaf(q[e], f[e], d);
#pragma unroll
            for (int x = 1; x < LPR; x <<= 1) d += __shfl_xor(d, x, kWave);
            sc[u] = real[u] ? d * scale : -INFINITY;
            mx = fmaxf(mx, sc[u]);
        }
        const float ref = mx == -INFINITY ? 0.f : mx, corr = __builtin_amdgcn_exp2f(m - ref);
        m = mx;
        sum *= corr;
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] *= corr;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[VE];
            row_piece<BF16>(vr[u], f);
            const float w = __builtin_amdgcn_exp2f(sc[u] - ref);
            sum += w;
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = fmaf(w, f[e], o[e]);
        }
    }
    // the row groups hold every RG-th key each
    float all = m;
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) all = fmaxf(all, __shfl_xor(all, x, kWave));
    const float ref = all == -INFINITY ? 0.f : all, corr = __builtin_amdgcn_exp2f(m - ref);
    sum *= corr;
#pragma unroll
    for (int e = 0; e < VE; ++e) o[e] *= corr;
#pragma unroll
    for (int x = LPR; x < kWave; x <<= 1) {
        sum += __shfl_xor(sum, x, kWave);
#pragma unroll
        for (int e = 0; e < VE; ++e) o[e] += __shfl_xor(o[e], x, kWave);
    }
    if (rg != 0) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;     // nothing seen: zeros
    uint4 w;
    if constexpr (BF16)
        w = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv), pack_bf16(o[4] * inv, o[5] * inv),
                       pack_bf16(o[6] * inv, o[7] * inv));
    else
        w = make_uint4(__float_as_uint(o[0] * inv), __float_as_uint(o[1] * inv), __float_as_uint(o[2] * inv), __float_as_uint(o[3] * inv));
    *(uint4*)(p.out + p.os.l * l + p.os.h * h + p.os.n * t + sub * 16) = w;
    if (!PAGED && sub == 0) p.lse[(int64_t)p.L * p.H * first + (int64_t)(l * p.H + h) * n + i] = kLn2 * (all + __builtin_amdgcn_logf(sum));
}

size_t packed_attn_ws_bytes(const pkv_packed&, int) { return 0; }

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
    const dim3 grid((unsigned)s.T, (unsigned)((s.H + 3) / 4), (unsigned)s.L);
#define PKV_ROWS(BF16, D, PAGED) hipLaunchKernelGGL((attn_rows_kernel<BF16, D, PAGED>), grid, dim3(256), 0, st, p)
    if (s.dtype == PKV_F32) {
        if (s.D == 128) PKV_ROWS(false, 128, true); else PKV_ROWS(false, 64, true);
    } else if (paged) {
        if (s.D == 128) PKV_ROWS(true, 128, true); else PKV_ROWS(true, 64, true);
    } else {
        if (s.D == 128) PKV_ROWS(true, 128, false); else PKV_ROWS(true, 64, false);
    }
#undef PKV_ROWS
    return hipGetLastError();
}

}  // namespace pkv
