// Launchers of the operators for packed prompts and paged caches, next to the others' (pkv_common.hpp).
#pragma once

#include "pkv_common.hpp"

namespace pkv {

constexpr int kMaxS = 4096;        // sequences of a packed call
constexpr int kMaxT = 1 << 22;     // rows of a packed call

hipError_t launch_compact_paged(const pkv_shape& s, const void* k, Strides ks, const void* v, Strides vs, const int32_t* order,
                                const int32_t* lengths, const pkv_paging& g, int l0, const int32_t* table, void* kp, void* vp,
                                int32_t* kept_pos, hipStream_t st);

// page operators: row_off is NULL for a resize (then target, and no slots), else target is NULL
size_t page_ws_bytes(int S, int layers);
hipError_t launch_pages(int S, int T, const pkv_paging& g, const int32_t* target, const int32_t* row_off, const int32_t* lens,
                        int32_t* table, int32_t* ring, const int32_t* state, int32_t* lens_out, int32_t* state_out,
                        int64_t* slots, int32_t* status, void* ws, hipStream_t st);

// v, slots and paging are NULL for a rotation without a store (then k_out, else kp and vp)
hipError_t launch_rope(const pkv_packed& s, const pkv_rope& r, const int32_t* pos, const void* q, Strides qs, const void* k,
                       Strides ks, const void* v, Strides vs, void* q_out, Strides qos, void* k_out, Strides kos,
                       const int64_t* slots, const pkv_paging* g, void* kp, void* vp, hipStream_t st);

// Rows of packed sequences and the keys they attend to: packed rows themselves (k, v; table NULL) or the pages.
struct PackedAttn {
    const void *q, *k, *v;
    Strides qs, ks, vs, os;
    const int32_t *row_off, *table, *lens;
    const float* scale;
    void* out;
    float* lse;           // packed prompts only
    pkv_paging g;
    int l0, max_rows;     // max_rows 0: packed prompts
    void* ws;
};
bool packed_attn_fits(const pkv_packed& s, const pkv_paging* g);
size_t packed_attn_ws_bytes(const pkv_packed& s, int max_rows);
hipError_t launch_packed_attn(const pkv_packed& s, const PackedAttn& a, hipStream_t st);

}  // namespace pkv
