// The 256-row attention kernel over 8-bit pools: see pv_attn_tile256.h.
#include "pv_attn_tile256.h"

namespace pv {

hipError_t launch_attn_kv8_tile256(const pv_plan *plan, const DeviceLists &dl, const void *q,
                                   const pv_kv8_pool &pool, const int32_t *page_table, float scale,
                                   void *out, float *ws_o, float *ws_ml, hipStream_t stream)
{
    return launch_tile256<true>(plan, dl, q, pool.k, pool.v, pool.k_scales, pool.v_scales, page_table,
                                scale, out, ws_o, ws_ml, stream);
}

}  // namespace pv
