// Rotary positions over several axes: pair i of the first rot columns of a row turns by pos[axis_i, t] * freq_i.
//
// The frequency is a fraction of a turn in units of 2^-64, so position * frequency modulo 2^64 is the angle modulo a turn
// without any loss, however far out the position is (in fp32 an angle of 10^6 radians is off by 0.03).  Its upper 32 bits
// are split into the nearest quarter turn and a rest of at most pi/4, for which the Taylor sums of sine and cosine up to x^9
// and x^10 are exact to fp32 (the first terms left out are below 2e-9).
// Bound: HBM; every row is read once and written once, in 16-byte pieces.  A lane has both columns of its pairs: two pieces
// of a row, half the rotated columns apart (or side by side if interleaved), a row is D*esize/32 lanes.  The sines are a
// token's, not a head's: a lane works out those of its pairs once and takes a group of heads through them.  The first head's row is
// asked for in front of the sines and every further one ahead of its turn (37.1 us -> 36.6; fp32, a head per lane, 7.5 -> 6.9).  5440
// tokens of 64 heads, D 128: 36.6 us for 178 MB read and written, 4.9 TB/s; a copy of that size runs at 4.6 to 5.0.
#include "packed.hpp"
#include "fast_div.hpp"

namespace pkv {

struct RopeParams {
    int T, H, Hkv;
    int group;                 // heads that a lane takes one after the other: query heads, key heads, with a store also value heads
    int num_pages, shift, axes;
    const uint64_t* freq;
    const int32_t* axis;
    const int32_t* pos;
    const unsigned char *q, *k, *v;
    unsigned char *q_out, *k_out;
    Strides qs, ks, vs, qos, kos;    // in bytes
    const int64_t* slots;
    unsigned char *kp, *vp;
};

// sine and cosine of `turns` / 2^32 of a turn
__device__ __forceinline__ void sin_cos_turn(uint32_t turns, float& sn, float& cs) {
    const uint32_t quarter = (turns + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turns - (quarter << 30)) * 1.4629180792671596e-9f;     // 2 pi / 2^32
    const float y = x * x;
    const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
    const bool odd = quarter & 1u;
    const float a = odd ? c : s, b = odd ? s : c;
    sn = (quarter & 2u) ? -a : a;
    cs = ((quarter + 1u) & 2u) ? -b : b;
}

// A row is read once: its lines need not stay (178 MB of rows: 42.7 us -> 37.1; stores past the caches too would be no faster, and
// the attention behind reads what is stored).
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const unsigned char* p) {
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4_t*)p));
}

template <bool BF16>
__device__ __forceinline__ void unpack_piece(const uint4& r, float* f) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        if constexpr (BF16) { f[2 * x] = __uint_as_float(w[x] << 16); f[2 * x + 1] = __uint_as_float(w[x] & 0xffff0000u); }
        else f[x] = __uint_as_float(w[x]);
    }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack_piece(const float* f) {
    if constexpr (BF16) return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// LPR lanes per row (D * esize / 32); half = pieces of half the rotated columns
template <bool BF16, int LPR, bool INTER, bool STORE>
__global__ void __launch_bounds__(256)
rope_kernel(RopeParams p, int half) {
    constexpr int VE = BF16 ? 8 : 4;                   // elements of a piece = pairs of a lane
    const int t = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, c = threadIdx.x % LPR;
    if (t >= p.T) return;
    const int h0 = blockIdx.y * p.group, l = blockIdx.z;
    const int all = p.H + (STORE ? 2 : 1) * p.Hkv, h1 = min(all, h0 + p.group);
    // the two pieces of this lane: a pair of rotated ones, or two of those behind them
    const bool turns = c < half;
    const int pa = INTER || !turns ? 2 * c : c, pb = INTER || !turns ? 2 * c + 1 : c + half;
    auto row_of = [&](int h) -> const unsigned char* {
        if (h < p.H) return p.q + p.qs.l * l + p.qs.h * h + p.qs.n * t;
        const bool val = STORE && h >= p.H + p.Hkv;
        const int g = h - p.H - (val ? p.Hkv : 0);
        return val ? p.v + p.vs.l * l + p.vs.h * g + p.vs.n * t : p.k + p.ks.l * l + p.ks.h * g + p.ks.n * t;
    };
    const unsigned char* first = row_of(h0);            // (rows of all heads are there to be read, whatever their slots)
    uint4 na = load_once(first + pa * 16), nb = load_once(first + pb * 16);
    float sn[VE], cs[VE];
    if (turns && h0 < p.H + p.Hkv) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const int i = c * VE + e;
            const uint32_t a = (uint32_t)p.axis[i];
            const int64_t pos = p.pos[(int64_t)(a < (uint32_t)p.axes ? a : 0u) * p.T + t];
            const uint64_t angle = (uint64_t)pos * p.freq[i];
            sin_cos_turn((uint32_t)((angle + 0x80000000ull) >> 32), sn[e], cs[e]);
        }
    }
    int64_t dst = -1;
    if constexpr (STORE) {
        if (h1 > p.H) {
            const int64_t slot = p.slots[(int64_t)l * p.T + t];
            if (slot >= 0 && (slot >> p.shift) < p.num_pages)
                dst = (((slot >> p.shift) * p.Hkv) << p.shift) + (slot & ((1 << p.shift) - 1));   // row of head 0
        }
    }
    constexpr int kRow = LPR * 32;                     // bytes of a row
    for (int h = h0; h < h1; ++h) {
        uint4 ra = na, rb = nb;
        if (h + 1 < h1) {
            const unsigned char* src = row_of(h + 1);
            na = load_once(src + pa * 16); nb = load_once(src + pb * 16);
        }
        unsigned char* to;
        if (h < p.H) {
            to = p.q_out + p.qos.l * l + p.qos.h * h + p.qos.n * t;
        } else {
            const bool val = STORE && h >= p.H + p.Hkv;
            const int g = h - p.H - (val ? p.Hkv : 0);
            if constexpr (STORE) {
                if (dst < 0) continue;
                to = (val ? p.vp : p.kp) + (dst + ((int64_t)g << p.shift)) * kRow;
            } else {
                to = p.k_out + p.kos.l * l + p.kos.h * g + p.kos.n * t;
            }
        }
        if (turns && h < p.H + p.Hkv) {
            float a[VE], b[VE];
            unpack_piece<BF16>(ra, a);
            unpack_piece<BF16>(rb, b);
            if constexpr (INTER) {
                // pairs are neighbours: those of the first piece, then those of the second
#pragma unroll
                for (int e = 0; e < VE; e += 2) {
                    const float x = a[e], y = a[e + 1], u = b[e], w = b[e + 1];
                    a[e] = x * cs[e / 2] - y * sn[e / 2];
                    a[e + 1] = y * cs[e / 2] + x * sn[e / 2];
                    b[e] = u * cs[VE / 2 + e / 2] - w * sn[VE / 2 + e / 2];
                    b[e + 1] = w * cs[VE / 2 + e / 2] + u * sn[VE / 2 + e / 2];
                }
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float x = a[e], y = b[e];
                    a[e] = x * cs[e] - y * sn[e];
                    b[e] = y * cs[e] + x * sn[e];
                }
            }
            ra = pack_piece<BF16>(a);
            rb = pack_piece<BF16>(b);
        }
        *(uint4*)(to + pa * 16) = ra;
        *(uint4*)(to + pb * 16) = rb;
    }
}

template <bool BF16, int LPR>
static void launch_rope_s(const RopeParams& p, int half, bool inter, bool store, dim3 grid, hipStream_t st) {
    if (inter) {
        if (store) hipLaunchKernelGGL((rope_kernel<BF16, LPR, true, true>), grid, dim3(256), 0, st, p, half);
        else hipLaunchKernelGGL((rope_kernel<BF16, LPR, true, false>), grid, dim3(256), 0, st, p, half);
    } else {
        if (store) hipLaunchKernelGGL((rope_kernel<BF16, LPR, false, true>), grid, dim3(256), 0, st, p, half);
        else hipLaunchKernelGGL((rope_kernel<BF16, LPR, false, false>), grid, dim3(256), 0, st, p, half);
    }
}

hipError_t launch_rope(const pkv_packed& s, const pkv_rope& r, const int32_t* pos, const void* q, Strides qs, const void* k,
                       Strides ks, const void* v, Strides vs, void* q_out, Strides qos, void* k_out, Strides kos,
                       const int64_t* slots, const pkv_paging* g, void* kp, void* vp, hipStream_t st) {
    const int esize = s.dtype == PKV_F32 ? 4 : 2;
    auto bytes = [esize](Strides x) { return Strides{0, x.l * esize, x.h * esize, x.n * esize}; };
    RopeParams p;
    p.T = s.T; p.H = s.H; p.Hkv = s.Hkv;
    p.num_pages = g ? g->num_pages : 0; p.shift = g ? __builtin_ctz((unsigned)g->page_size) : 0; p.axes = r.axes;
    p.freq = r.freq; p.axis = r.axis; p.pos = pos;
    p.q = (const unsigned char*)q; p.k = (const unsigned char*)k; p.v = (const unsigned char*)v;
    p.q_out = (unsigned char*)q_out; p.k_out = (unsigned char*)k_out;
    p.qs = bytes(qs); p.ks = bytes(ks); p.vs = bytes(vs); p.qos = bytes(qos); p.kos = bytes(kos);
    p.slots = slots; p.kp = (unsigned char*)kp; p.vp = (unsigned char*)vp;
    const int lpr = s.D * esize / 32, all = s.H + (slots ? 2 : 1) * s.Hkv;
    const long long rows = (s.T + 256 / lpr - 1) / (256 / lpr);
    // Groups of up to eight heads share a token's sines while that leaves the chip four workgroups per compute unit.
    int group = 8;
    while (group > 1 && rows * s.L * ((all + group - 1) / group) < 4ll * compute_units()) group >>= 1;
    p.group = group;
    const dim3 grid((unsigned)rows, (unsigned)((all + group - 1) / group), (unsigned)s.L);
    const int half = r.rot_dim / 2 * esize / 16;
    const bool inter = r.interleaved != 0, store = slots != nullptr;
    if (s.dtype == PKV_BF16) {
        if (s.D == 128) launch_rope_s<true, 8>(p, half, inter, store, grid, st);
        else launch_rope_s<true, 4>(p, half, inter, store, grid, st);
    } else {
        if (s.D == 128) launch_rope_s<false, 16>(p, half, inter, store, grid, st);
        else launch_rope_s<false, 8>(p, half, inter, store, grid, st);
    }
    return hipGetLastError();
}

}  // namespace pkv
