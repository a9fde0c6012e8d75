// What the two 16-row attention kernels share: the end of an item (gfx950 only).
#pragma once

#include "pv_device.h"

namespace pv {

// Merges the (max, sum, O) triples of an item's NW wavefronts through LDS and writes its rows, to
// `out` or, for a part of a KV range, to the workspace.  Lane = (row q16, group g) holds O^T rows 16 *
// blk + 4 * g .. + 3 of its row in o[blk], the row's running maximum and its share of the sum.
template <typename T, int D, int NW>
__device__ __forceinline__ void finish_narrow_item(
    const WorkItem &it, int32_t group, int32_t num_q_heads, const f32x4 (&o)[D / 16], float m_run,
    float l_run, float (&sm_o)[NW][16][D + 4], float (&sm_m)[NW][16], float (&sm_l)[NW][16],
    uint16_t *__restrict__ out, float *__restrict__ ws_o, float *__restrict__ ws_ml)
{
    constexpr int NB = D / 16;
    const int lane = lane_id();
    const int w = wave_id();
    const int q16 = lane & 15;
    const int g = lane >> 4;
    float l_tot = l_run + __shfl_xor(l_run, 16);
    l_tot += __shfl_xor(l_tot, 32);
    if (g == 0) {
        sm_m[w][q16] = m_run;
        sm_l[w][q16] = l_tot;
    }
#pragma unroll
    for (int blk = 0; blk < NB; ++blk)
        *reinterpret_cast<f32x4 *>(&sm_o[w][q16][16 * blk + 4 * g]) = o[blk];
    __syncthreads();

    constexpr int THREADS = 4 * NW;    // of a row
    constexpr int PER = D / THREADS;   // output elements per thread
    const int r16 = (int)threadIdx.x / THREADS;
    const int d0 = ((int)threadIdx.x & (THREADS - 1)) * PER;
    if (r16 >= it.row_count) return;
    float mw[NW], wgt[NW];
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        mw[i] = sm_m[i][r16];
        M = fmaxf(M, mw[i]);
    }
    const float M_safe = M == -INFINITY ? 0.f : M;
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        wgt[i] = fast_exp2(mw[i] - M_safe);
        L += wgt[i] * sm_l[i][r16];
    }
    float acc[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) a += wgt[i] * sm_o[i][r16][d0 + e];
        acc[e] = a;
    }
    const int orow = it.row_begin + r16;
    if (it.split_count == 1) {
        const float inv = 1.f / L;
        const int otok = orow / group;
        const int ohq = it.kv_head * group + orow % group;
        uint16_t *dst = out + ((int64_t)(it.q_row0 + otok) * num_q_heads + ohq) * D + d0;
        uint32_t packed[PER / 2];
#pragma unroll
        for (int e = 0; e < PER / 2; ++e)
            packed[e] = T::pack2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
        if constexpr (PER == 8) {
            *reinterpret_cast<u32x4 *>(dst) = u32x4{packed[0], packed[1], packed[2], packed[3]};
        } else if constexpr (PER == 2) {
            *reinterpret_cast<uint32_t *>(dst) = packed[0];
        } else {
            *reinterpret_cast<u32x2 *>(dst) = u32x2{packed[0], packed[1]};
        }
    } else {
        const int64_t slot = (int64_t)it.partial_base + r16;
        float *po = ws_o + slot * D + d0;
        if constexpr (PER == 2) {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            *reinterpret_cast<f32x2 *>(po) = f32x2{acc[0], acc[1]};
        } else {
#pragma unroll
            for (int e = 0; e < PER; e += 4)
                *reinterpret_cast<f32x4 *>(po + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        }
        if (d0 == 0) {
            ws_ml[2 * slot] = M;
            ws_ml[2 * slot + 1] = L;
        }
    }
}

}  // namespace pv
