// quant4.h -- shared by the kernels of the 4-bit KV cache (quant4_*.hip), by
// the reading back of both caches (quant_read.hip) and by their entry points
// (quant_api.hip) (not part of the C ABI).
#pragma once
#include "quant.h"

namespace mosaic {

// The cache's tensors (mosaic_nibble_cache), passed by value.
struct Q4Cache {
    int S, H, G, N;                                        // sequences, kv heads, group, blocks of a pair at most
    int cap;                                               // tokens of a sequence at most
    uint8_t *k, *v;                                        // codes [S][H][N][B][D / 2] and [S][H][N][D][B / 2]
    uint16_t *kg, *vg;                                     // scales and zeros [S][H][N][2][D] and [S][H][N][2][B]
    uint16_t *kt, *vt;                                     // unfinished block [S][H][B][D] and [S][H][D][B]
    int32_t *lens;                                         // as in QCache
    int32_t *arrivals;
    int32_t *refused;
    __device__ __forceinline__ int len(long long p) const { return min(max(lens[p], 0), cap); }
};

// where a run of tokens is read back to, strides in elements
struct QOut {
    uint16_t *k, *v;
    int64_t k_seq, k_head, k_tok, v_seq, v_head, v_tok;
    const int32_t *starts;                                 // [S] on the device, or null: start
    int start, n;
};

// several query tokens of a sequence, and their outputs; strides in elements
struct QChunk {
    const uint16_t *q;
    uint16_t *out;
    int64_t q_seq, q_tok, q_head, o_seq, o_tok, o_head;
    const int32_t *counts;                                 // [S] on the device, or null: n each
    int n, causal;
    float scale;
};

// least scale of a grid, as a 16-bit pattern: 2^-19 of fp16 (its numbers below
// have too few bits: codes reach 15.5 of a smaller scale), 2^-100 of bf16
template <int DT> __device__ constexpr uint32_t q4_least() { return DT ? 27u << 7 : 32u; }

// two fp32 values rounded to the element type (to nearest even; NaN stays NaN)
template <int DT> __device__ __forceinline__ uint32_t pack16(float a, float b) {
    if constexpr (DT) {
        typedef __attribute__((ext_vector_type(2))) __bf16 b2;
        b2 r;
        r[0] = (__bf16)a;
        r[1] = (__bf16)b;
        return __builtin_bit_cast(uint32_t, r);
    } else {
        typedef __attribute__((ext_vector_type(2))) _Float16 h2;
        h2 r;
        r[0] = (_Float16)a;
        r[1] = (_Float16)b;
        return __builtin_bit_cast(uint32_t, r);
    }
}
// The softmax scale in powers of two, positive (a negative one's sign goes to the
// query), as logits are scaled when their maximum is known.  A scale of zero is one
// of a query of zeros: a masked logit, minus infinity, times zero would be NaN.
__device__ __forceinline__ float powers_of(float scale) { return scale == 0.0f ? 1.0f : fabsf(scale) * 1.44269504088896340736f; }
__device__ __forceinline__ uint32_t flip_of(float scale) { return scale < 0.0f ? 0x80008000u : 0u; }
// element i of 16-bit pairs
template <int DT> __device__ __forceinline__ float half_of(const uint32_t *w, int i) {
    return h2f((uint16_t)((i & 1) ? w[i >> 1] >> 16 : w[i >> 1]), DT);
}

// ---------------------------------------------------------------- launchers
hipError_t launch_quant4_append(const Q4Cache &q, int block, int dtype, const QNew &n, hipStream_t s);
size_t quant4_attn_ws_bytes(int pairs);
hipError_t launch_quant4_attn(const Q4Cache &q, int block, int dtype, const uint16_t *query, float scale, void *ws, float *out,
                              hipStream_t s);
size_t quant4_chunk_ws_bytes(int pairs, int blocks, int block);
hipError_t launch_quant4_chunk(const Q4Cache &q, int block, int dtype, const QChunk &c, float *part, hipStream_t s);
hipError_t launch_quant4_read(const Q4Cache &q, int block, int dtype, const QOut &o, hipStream_t s);
hipError_t launch_quant_read(const QCache &q, int fmt, int block, int dtype, const QOut &o, hipStream_t s);

}  // namespace mosaic
