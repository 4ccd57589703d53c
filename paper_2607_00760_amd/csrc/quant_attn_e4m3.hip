// quant_attn_e4m3.hip -- attention over the 8-bit KV cache, E4M3 codes.
#include "quant_attn.h"

namespace mosaic {

hipError_t launch_quant_attn_e4m3(const QCache &q, int block, int dtype, const uint16_t *query, float scale, const QSel &sel,
                                  void *ws, float *out, hipStream_t s) {
    return launch_quant_attn_t<QF_E4M3>(q, block, dtype, query, scale, sel, ws, out, s);
}

size_t quant_attn_ws_bytes(int pairs) {
    return (size_t)2 * Q_RUNS * sizeof(uint32_t) + (size_t)(qa_runs(pairs) + pairs) * QA_PART * sizeof(float);
}

}  // namespace mosaic
