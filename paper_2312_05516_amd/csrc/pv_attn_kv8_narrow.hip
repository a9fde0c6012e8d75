// Bandwidth-oriented attention kernel over 8-bit pools: work items of at most 16 query rows.
//
// What attn_narrow_kernel computes, over K, V = code * 2^e (see pv_kv8.h).  Codes become 16-bit
// values in registers, by one conversion for two of them that takes the page's scale along, and
// nothing is rounded by that: the result is that of 16-bit attention over the values that reading the
// pools back would give.
//
// Mapping to gfx950.  One workgroup = 4 wavefronts (8 in short lists, see pv_plan::narrow_eight) = one
// item; the wavefronts take the 64-key blocks (four pages) of the item round-robin, two blocks' loads in
// flight, nothing is shared until the end.
// A lane's 16 bytes are 16 codes: of K 16 dimensions of one slot, two operands of
// v_mfma_f32_16x16x32 (S^T = K Q^T, the dimensions contracted in that order); of V the 16 slots of
// one dimension.  S^T row 4g + i of the b-th of a block's four score tiles is fed with slot 4b + i of
// its g-th page, so that lane group g holds the scores of the whole page g, 16 keys in order: the
// operand for the 16 slots that its lanes hold of V.
//
// What bounds it: HBM.  Blocks are 64 keys because a lane's 16 bytes of V are 16 keys and four lane groups
// share a block; page ids come a block before the loads that need them, codes are read with the streaming
// hint (8-10 % of a large list).  96 generation steps over 0.5-4 K keys, 40/40 heads: 2.32 GB in 346 us =
// 6.7 TB/s, what reads alone reach; 64 over 0.1-6 K, 64/8 heads: 388 MB in 66 us = 5.9 TB/s, the rest the
// set-up of items (three dependent round trips) and the tail of the launch.
#include "pv_kv8.h"
#include "pv_narrow.h"

namespace pv {

template <int D>
struct Narrow8Frag {
    u32x4 k[4][D / 64];  // [score tile][64 dimensions]
    u32x4 v[D / 16];     // [16-wide block of d]
    uint32_t k_scale, v_scale;
};

template <typename T, int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void attn_kv8_narrow_kernel(
    const WorkItem *__restrict__ items, const uint16_t *__restrict__ q, Kv8Ptrs pool,
    const int32_t *__restrict__ page_table, int32_t max_pages, int32_t num_q_heads,
    int32_t num_kv_heads, int32_t group, float scale_log2e, uint16_t *__restrict__ out,
    float *__restrict__ ws_o, float *__restrict__ ws_ml)
{
    constexpr int BK = 64;
    constexpr int JJ = D / 64;
    constexpr int NB = D / 16;
    typedef typename T::vec8 vec8;
    __shared__ float sm_o[NW][16][D + 4];
    __shared__ float sm_m[NW][16];
    __shared__ float sm_l[NW][16];

    const WorkItem it = items[blockIdx.x];
    const int lane = lane_id();
    const int w = wave_id();
    const int q16 = lane & 15;
    const int g = lane >> 4;

    const int row = it.row_begin + q16;
    const bool valid = q16 < it.row_count;
    const int tok = valid ? row / group : 0;
    const int hq = it.kv_head * group + (valid ? row % group : 0);
    // one past the last key of the item that this row may see (rows beyond the item are fed zeros, any
    // limit works); a part of a KV range may end inside a block
    const int vis_end = valid ? min(it.ctx + tok + 1, it.kv_end) : it.kv_end;
    // every valid row sees all keys below this
    const int unmasked_end = min(it.ctx + it.row_begin / group + 1, it.kv_end);

    vec8 qf[2 * JJ];
    {
        const uint16_t *qrow = q + ((int64_t)(it.q_row0 + tok) * num_q_heads + hq) * D;
#pragma unroll
        for (int i = 0; i < 2 * JJ; ++i) {
            u32x4 raw = {0u, 0u, 0u, 0u};
            if (valid) raw = load16(qrow + 64 * (i / 2) + 16 * g + 8 * (i % 2));
            qf[i] = as_vec8<T>(raw);
        }
    }

    const int32_t *pt = page_table + (int64_t)it.req * max_pages;
    const int last_pg = (it.kv_end - 1) >> 4;
    const int pg0 = it.kv_begin >> 4;
    const int nblocks = (it.kv_end - it.kv_begin + BK - 1) / BK;
    const int k_page = q16 >> 2;                        // page of a block that the lane reads K of
    const int k_at = g * 64 + (q16 & 3) * 16;           // + tile * 4 * D + 64 dimensions * 256
    const int v_at = q16 * 16;                          // + blk * 256

    // page ids of a block, fetched a block before its K and V so that these do not wait for them
    int ids[4];
    auto page_ids = [&](int b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ids[i] = pt[min(pg0 + 4 * b + i, last_pg)];
    };
    auto load_block = [&](Narrow8Frag<D> &f, int b) {
        int64_t tile[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[i] = (int64_t)ids[i] * num_kv_heads + it.kv_head;
        page_ids(b + NW);
        const int64_t k01 = k_page & 1 ? tile[1] : tile[0], k23 = k_page & 1 ? tile[3] : tile[2];
        const int64_t v01 = g & 1 ? tile[1] : tile[0], v23 = g & 1 ? tile[3] : tile[2];
        const int64_t kt = k_page & 2 ? k23 : k01, vt = g & 2 ? v23 : v01;
        const uint8_t *kb = pool.k + kt * (16 * D) + k_at;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < JJ; ++j) f.k[t][j] = load16_stream(kb + t * (4 * D) + j * 256);
        f.k_scale = pool.k_scales[kt];
        const uint8_t *vb = pool.v + vt * (16 * D) + v_at;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) f.v[blk] = load16_stream(vb + blk * 256);
        f.v_scale = pool.v_scales[vt];
    };

    f32x4 o[NB];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) o[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY;  // running maximum of the scaled scores (log2 domain)
    float l_run = 0.f;        // this lane's share of the running sum
    uint32_t any_nan = 0;     // whether NaNs were left out of a masked block

    auto compute_block = [&](Narrow8Frag<D> &f, int b) {
        const int kb0 = it.kv_begin + BK * b;
        const float k_scale = exp2_scale((int)f.k_scale), v_scale = exp2_scale((int)f.v_scale);
        float x[16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < JJ; ++j) {
                const u32x4 c = f.k[t][j];
                s = T::mfma16(as_vec8<T>(decode8<T>(c[0], c[1], k_scale)), qf[2 * j], s);
                s = T::mfma16(as_vec8<T>(decode8<T>(c[2], c[3], k_scale)), qf[2 * j + 1], s);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * t + i] = s[i] * scale_log2e;
        }
        if (kb0 + BK > unmasked_end) {  // block reaches the causal boundary or the end
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (kb0 + 16 * g + j >= vis_end) x[j] = -INFINITY;
        }
        if (kb0 + BK > unmasked_end) {
            // Slots past the end may hold anything: no V codes there.  Nor NaNs among values that some
            // row does not see: zero times them would be NaN in that row too; see below.
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t mask = codes_in_front(it.kv_end - kb0 - 16 * g - 4 * i);
#pragma unroll
                for (int blk = 0; blk < NB; ++blk) {
                    const uint32_t codes = f.v[blk][i] & mask;
                    const uint32_t nan = nan_codes(codes);
                    any_nan |= nan;
                    f.v[blk][i] = codes & ~((nan >> 7) * 0xFFu);
                }
            }
        }
        float mx = x[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = fmaxf(mx, x[j]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run, mx);
        const float m_safe = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2(m_run - m_safe);
        m_run = m_new;
        float psum = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            x[j] = fast_exp2(x[j] - m_safe);
            psum += x[j];
        }
        l_run = l_run * alpha + psum;
        if (__any(alpha != 1.f)) {
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) o[blk] *= alpha;
        }
        // The probabilities are rounded to 16 bits for the product with V, their sum is not: results are
        // 1.8e-3 from 64 bits in bf16 (relative 2-norm; the rounding of the result alone 1.66e-3), and 6 %
        // of the time of short lists would buy a second term that takes that back.
        u32x4 p[2];
#pragma unroll
        for (int jj = 0; jj < 8; ++jj) p[jj / 4][jj % 4] = T::pack2(x[2 * jj], x[2 * jj + 1]);
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            const u32x4 c = f.v[blk];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const vec8 v = as_vec8<T>(decode8<T>(c[2 * half], c[2 * half + 1], v_scale));
                o[blk] = T::mfma16(v, as_vec8<T>(p[half]), o[blk]);
            }
        }
    };

    {
        Narrow8Frag<D> fa, fb;
        int b = w;
        page_ids(b);
        if (b < nblocks) load_block(fa, b);
        while (b < nblocks) {
            int nxt = b + NW;
            if (nxt < nblocks) load_block(fb, nxt);
            compute_block(fa, b);
            b = nxt;
            if (b >= nblocks) break;
            nxt = b + NW;
            if (nxt < nblocks) load_block(fa, nxt);
            compute_block(fb, b);
            b = nxt;
        }
    }
    // NaNs that were left out belong into the rows that see them: counted for each row and dimension by
    // one more product, of ones in their places with ones for the keys that a row sees.
    if (__any(any_nan != 0)) {
#pragma unroll 1
        for (int b = w; b < nblocks; b += NW) {
            const int kb0 = it.kv_begin + BK * b;
            if (kb0 + BK <= unmasked_end) continue;
            u32x4 seen[2];
#pragma unroll
            for (int jj = 0; jj < 8; ++jj) {
                const int key = kb0 + 16 * g + 2 * jj;
                seen[jj / 4][jj % 4] =
                    T::pack2(key < vis_end ? 1.f : 0.f, key + 1 < vis_end ? 1.f : 0.f);
            }
            const int64_t tile =
                (int64_t)pt[min(pg0 + 4 * b + g, last_pg)] * num_kv_heads + it.kv_head;
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) {
                u32x4 bad = load16(pool.v + tile * (16 * D) + v_at + blk * 256);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    bad[i] = (nan_codes(bad[i] & codes_in_front(it.kv_end - kb0 - 16 * g - 4 * i)) >> 7) *
                             0x38u;  // the code of 1
                f32x4 n = {0.f, 0.f, 0.f, 0.f};
                n = T::mfma16(as_vec8<T>(decode8<T>(bad[0], bad[1], 1.f)), as_vec8<T>(seen[0]), n);
                n = T::mfma16(as_vec8<T>(decode8<T>(bad[2], bad[3], 1.f)), as_vec8<T>(seen[1]), n);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[blk][i] = n[i] > 0.f ? NAN : o[blk][i];
            }
        }
    }
    finish_narrow_item<T, D, NW>(it, group, num_q_heads, o, m_run, l_run, sm_o, sm_m, sm_l, out, ws_o,
                             ws_ml);
}

template <typename T, int D>
static void launch_kv8_narrow_t(const pv_plan *plan, const DeviceLists &dl, const void *q,
                                const Kv8Ptrs &pool, const int32_t *page_table, float scale,
                                void *out, float *ws_o, float *ws_ml, hipStream_t stream)
{
    auto kernel = plan->narrow_eight ? attn_kv8_narrow_kernel<T, D, 8> : attn_kv8_narrow_kernel<T, D, 4>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan->narrow.size()),
                       dim3(plan->narrow_eight ? 512 : 256), 0, stream, dl.narrow, (const uint16_t *)q, pool, page_table, plan->max_pages_per_req,
                       plan->num_q_heads, plan->pool.num_kv_heads, plan->group, scale * kLog2e,
                       (uint16_t *)out, ws_o, ws_ml);
}

hipError_t launch_attn_kv8_narrow(const pv_plan *plan, const DeviceLists &dl, const void *q,
                                  const pv_kv8_pool &pool, const int32_t *page_table, float scale,
                                  void *out, float *ws_o, float *ws_ml, hipStream_t stream)
{
    if (plan->narrow.empty()) return hipSuccess;
    const bool h = plan->pool.dtype == PV_F16;
    const Kv8Ptrs p = {static_cast<uint8_t *>(pool.k), static_cast<uint8_t *>(pool.v), pool.k_scales,
                       pool.v_scales};
    auto go = plan->pool.head_dim == 128
                  ? (h ? launch_kv8_narrow_t<F16, 128> : launch_kv8_narrow_t<BF16, 128>)
                  : (h ? launch_kv8_narrow_t<F16, 64> : launch_kv8_narrow_t<BF16, 64>);
    go(plan, dl, q, p, page_table, scale, out, ws_o, ws_ml, stream);
    return hipGetLastError();
}

}  // namespace pv
