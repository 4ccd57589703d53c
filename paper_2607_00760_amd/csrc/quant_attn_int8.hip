// quant_attn_int8.hip -- attention over the 8-bit KV cache, 8-bit integer codes.
#include "quant_attn.h"

namespace mosaic {

hipError_t launch_quant_attn_int8(const QCache &q, int block, int dtype, const uint16_t *query, float scale, const QSel &sel,
                                  void *ws, float *out, hipStream_t s) {
    return launch_quant_attn_t<QF_INT8>(q, block, dtype, query, scale, sel, ws, out, s);
}

}  // namespace mosaic
