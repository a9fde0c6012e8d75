// The 256-row attention kernel over 16-bit pools: see pv_attn_tile256.h.
#include "pv_attn_tile256.h"

namespace pv {

hipError_t launch_attn_tile256(const pv_plan *plan, const DeviceLists &dl, const void *q, const void *k_pages,
                               const void *v_pages, const int32_t *page_table, float scale,
                               void *out, float *ws_o, float *ws_ml, hipStream_t stream)
{
    return launch_tile256<false>(plan, dl, q, k_pages, v_pages, nullptr, nullptr, page_table, scale,
                                 out, ws_o, ws_ml, stream);
}

}  // namespace pv
