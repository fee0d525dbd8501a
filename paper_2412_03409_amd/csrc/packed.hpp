// Launchers of the operators for packed prompts and paged caches, next to the others' (pkv_common.hpp).
#pragma once

#include "pkv_common.hpp"

namespace pkv {

constexpr int kMaxS = 4096;        // sequences of a packed call
constexpr int kMaxT = 1 << 22;     // rows of a packed call
constexpr int kMaxBeams = 32;      // of a prompt
constexpr int kMaxPieces = 64;     // of a row of logits
constexpr int kMaxV = 1 << 20;     // tokens: 64 pieces of 16384

hipError_t launch_compact_paged(const pkv_shape& s, const void* k, Strides ks, const void* v, Strides vs, const int32_t* order,
                                const int32_t* lengths, const pkv_paging& g, int l0, const int32_t* table, void* kp, void* vp,
                                int32_t* kept_pos, hipStream_t st);

// page operators: row_off is NULL for a resize (then target, and no slots), else target is NULL
size_t page_ws_bytes(int S, int layers);
hipError_t launch_pages(int S, int T, const pkv_paging& g, const int32_t* target, const int32_t* row_off, const int32_t* lens,
                        int32_t* table, int32_t* ring, const int32_t* state, int32_t* lens_out, int32_t* state_out,
                        int64_t* slots, int32_t* status, void* ws, hipStream_t st);

// places follow their beams: groups of W places
bool reorder_fits(int S, int W, int Hkv, int row_bytes, const pkv_paging& g);
size_t reorder_ws_bytes(int S, int layers);
hipError_t launch_reorder(int S, int W, int Hkv, int row_bytes, const pkv_paging& g, const int32_t* parents, const int32_t* table,
                          const int32_t* lens, int32_t* ring, const int32_t* state, int32_t* table_out, int32_t* lens_out,
                          int32_t* state_out, void* kp, void* vp, int32_t* status, void* ws, hipStream_t st);

// the best continuations of S prompts of W beams
size_t beam_ws_bytes(int S, int W, int V, int esize);
hipError_t launch_beam(int S, int W, int V, bool bf16, const void* logits, int64_t stride, const float* scores, const uint8_t* ended,
                       int end_token, int32_t* tokens, int32_t* parents, float* scores_out, uint8_t* ended_out, void* ws,
                       hipStream_t st);

// v, slots and paging are NULL for a rotation without a store (then k_out, else kp and vp)
hipError_t launch_rope(const pkv_packed& s, const pkv_rope& r, const int32_t* pos, const void* q, Strides qs, const void* k,
                       Strides ks, const void* v, Strides vs, void* q_out, Strides qos, void* k_out, Strides kos,
                       const int64_t* slots, const pkv_paging* g, void* kp, void* vp, hipStream_t st);

// Rows of packed sequences and the keys they attend to: packed rows themselves (k, v; table and state_off NULL), the pages, or
// states of another length (k, v; state_off).
struct PackedAttn {
    const void *q, *k, *v;
    Strides qs, ks, vs, os;
    const int32_t *row_off, *table, *lens;
    const float* scale;
    void* out;
    float* lse;           // packed prompts only
    pkv_paging g;
    int l0, max_rows;     // max_rows 0: packed prompts
    int M;                // states
    const int32_t *state_off, *seen;
    void* ws;
};
bool packed_attn_fits(const pkv_packed& s, const pkv_paging* g);
size_t packed_attn_ws_bytes(const pkv_packed& s, int max_rows);
bool cross_attn_fits(const pkv_packed& s, int M);
size_t cross_attn_ws_bytes(const pkv_packed& s, int M, int max_rows);
// ... of many bf16 rows over states
size_t cross_tiles_ws_bytes(const pkv_packed& s, int M);
hipError_t launch_cross_tiles(const pkv_packed& s, const PackedAttn& a, hipStream_t st);
hipError_t launch_packed_attn(const pkv_packed& s, const PackedAttn& a, hipStream_t st);

}  // namespace pkv
