// norm_rope.h -- the norm-and-rotation pass, between its kernel (norm_rope.hip)
// and its entry point (quant_api.hip) (not part of the C ABI).
#pragma once
#include "mosaic_internal.h"

namespace mosaic {

// queries, keys and (v set) values of `seqs` sequences of n tokens
struct NormRope {
    struct Part { const uint16_t *in; uint16_t *out; int64_t in_seq, in_tok, in_head, out_seq, out_tok, out_head; };
    Part q, k, vp;
    const uint16_t *qw, *kw;              // weights, or null: no norm
    const float *inv_freq;                // [half]
    const void *pos;
    int64_t pos_seq, pos_tok;
    int seqs, n, hq, hkv, half, pos64, v;
    float eps;
};
hipError_t launch_norm_rope(const NormRope &a, int dtype, int interleaved, hipStream_t s);

}  // namespace mosaic
