// Rotary position embedding fused with the KV append: the producer step in front of the hot path
// for the Llama 2 models of the paper (Section 6.1 lists rotary embedding among their features;
// Section 4.4.1: the linear layers produce each token's Q/K/V, the new K/V are stored in their
// slots, then attention runs).  One launch rotates the new K rows and stores them in the pool,
// stores the new V rows, and rotates the Q rows, instead of a rotary pass over Q and K followed by
// the append.
//
// The transform is the published RoFormer one: pair i of a head, for a token at logical position
// t, is rotated by t * theta_i.  cos / sin come from a table [max_pos][D] (D/2 cosines, then D/2
// sines) that the caller computes once (pv_rope_table).  Pairing: style 0 = elements (2i, 2i+1),
// style 1 = elements (i, i + D/2).  The rotation is evaluated in fp32 and rounded to the 16-bit
// type (nearest even); V is moved bit for bit.
//
// Grid: (append groups, head blocks) with D threads; a head block is HB heads of one kind, the KV
// heads first (K rotated + scattered, V scattered as in kv_append_kernel), then the query heads of
// the group's tokens.  The heads of a token share its angles, which are twice the bytes of one
// head's row, so a thread loads them once for all its heads, and then all its rows at once.
#include "pv_norm_rope.h"

namespace pv {

// NORM: rows whose kind has a weight are first scaled to y = x * w / sqrt(mean(x^2) + eps), in fp32
// and without a rounding of their own; the lanes that hold a row are neighbours.  Bound: HBM, as without.
// 6 prompts, 4.8 K tokens, 40/40 heads: 296 MB in 62.3 us = 4.8 TB/s (between calls).
//
// kVApart: V in workgroups of its own, in front of the others.  Behind K's norms and rotation its loads come
// late: the same 6 prompts 65.2 us otherwise, 63.0 so (half pairs 62.4 and 61.6, 64/8 heads the same; head
// size 64 1-2 % slower).
template <int D, int HB, bool NORM>
constexpr bool kVApart = NORM && HB > 1 && D == 128;

template <typename T, int D, int STYLE, int HB, bool NORM>
__global__ __launch_bounds__(D) void rope_append_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in,
    uint16_t *q_out /* may be q_in */, const uint16_t *__restrict__ k_new,
    const uint16_t *__restrict__ v_new, const float *__restrict__ cos_sin,
    const int32_t *__restrict__ page_table, int32_t max_pages, int32_t num_q_heads,
    int32_t num_kv_heads, uint16_t *__restrict__ k_pages, uint16_t *__restrict__ v_pages,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps)
{
    constexpr int CH = D / 8;
    const AppendGroup g = groups[blockIdx.x];
    const int kv_blocks = (num_kv_heads + HB - 1) / HB;
    constexpr bool V_APART = kVApart<D, HB, NORM>;
    const bool v_only = V_APART && (int)blockIdx.y < kv_blocks;
    const int y = (int)blockIdx.y - (V_APART && !v_only ? kv_blocks : 0);
    const int t = (int)threadIdx.x;
    const bool is_q = y >= kv_blocks;
    const int h0 = (is_q ? y - kv_blocks : y) * HB;
    const int heads = min(HB, (is_q ? num_q_heads : num_kv_heads) - h0);
    const int64_t row_stride = (int64_t)(is_q ? num_q_heads : num_kv_heads) * D;
    const int64_t src_off = (int64_t)g.q_row * row_stride + (int64_t)h0 * D;
    const uint16_t *src = (is_q ? q_in : k_new) + src_off;

    const uint16_t *weight = NORM ? (is_q ? q_weight : k_weight) : nullptr;
    // a lane's weights: of chunk c8 and, for pairs across the halves of a head, of its partner
    u32x4 weights[2];
    if (NORM && weight) {
        const int c8 = STYLE == 0 ? t % CH : t % (CH / 2);
        weights[0] = load16(weight + 8 * c8);
        if constexpr (STYLE == 1) weights[1] = load16(weight + D / 2 + 8 * c8);
    }

    int64_t tile = 0;
    int slot0 = 0;
    if (!is_q) {
        const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
        slot0 = g.t_begin & 15;
        tile = (page * num_kv_heads + h0) * (int64_t)(16 * D);
    }
    // destination of the 16-byte chunk c8 of token j, head i of the block
    auto store_chunk = [&](int j, int i, int c8, u32x4 val) {
        if (is_q)
            *reinterpret_cast<u32x4 *>(q_out + src_off + j * row_stride + i * D + 8 * c8) = val;
        else
            *reinterpret_cast<u32x4 *>(k_pages + tile + i * (16 * D) + (c8 * 16 + slot0 + j) * 8) =
                val;
    };

    if (v_only) {
        // below
    } else if constexpr (STYLE == 0) {
        // one thread per (token j, chunk c8): 4 pairs inside the chunk, of every head
        const int j = t / CH, c8 = t % CH;
        if (j < g.count) {
            const float *cs = cos_sin + (int64_t)(g.t_begin + j) * D;
            const f32x4 c = *reinterpret_cast<const f32x4 *>(cs + 4 * c8);
            const f32x4 s = *reinterpret_cast<const f32x4 *>(cs + D / 2 + 4 * c8);
            u32x4 raw[HB];
#pragma unroll
            for (int i = 0; i < HB; ++i)
                raw[i] = load16_as<(HB > 1)>(src + j * row_stride + (i < heads ? i : 0) * D + 8 * c8);
#pragma unroll
            for (int i = 0; i < HB; ++i) {
                float x[8], o[8];
                unpack8<T>(raw[i], x);
                if (NORM && weight) {
                    float w[8];
                    unpack8<T>(weights[0], w);
                    const float mine = sum_squares(x);
                    float partner;  // the chunk half a row away
                    if constexpr (D == 128)
                        partner = __builtin_bit_cast(
                            float, other_lane<8>(__builtin_bit_cast(uint32_t, mine)));
                    else
                        partner = __shfl_xor(mine, 4);
                    const float r = norm_factor<D>(mine + partner, eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * r * w[e];
                }
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    if constexpr (NORM) {
                        rotate_pair(x[2 * p], x[2 * p + 1], c[p], s[p], o[2 * p], o[2 * p + 1]);
                    } else {
                        o[2 * p] = x[2 * p] * c[p] - x[2 * p + 1] * s[p];
                        o[2 * p + 1] = x[2 * p + 1] * c[p] + x[2 * p] * s[p];
                    }
                }
                if (i < heads) store_chunk(j, i, c8, pack8<T>(o));
            }
        }
    } else {
        // one thread per (token j, chunk c8 of the first half): its partner chunk is c8 + CH/2.  A
        // head takes half of the threads; with several heads the other half takes every other one.
        constexpr int LANES = 8 * (CH / 2);
        constexpr int SIDES = HB > 1 ? 2 : 1;
        constexpr int MINE = HB / SIDES;
        const int side = t / LANES, j = t % LANES / (CH / 2), c8 = t % (CH / 2);
        if (side < SIDES && j < g.count) {
            const float *cs = cos_sin + (int64_t)(g.t_begin + j) * D;
            f32x4 c[2], s[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                c[half] = *reinterpret_cast<const f32x4 *>(cs + 8 * c8 + 4 * half);
                s[half] = *reinterpret_cast<const f32x4 *>(cs + D / 2 + 8 * c8 + 4 * half);
            }
            u32x4 ra[MINE], rb[MINE];
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const int i = SIDES * m + side;
                const uint16_t *row = src + j * row_stride + (i < heads ? i : 0) * D + 8 * c8;
                ra[m] = load16_as<(HB > 1)>(row);
                rb[m] = load16_as<(HB > 1)>(row + D / 2);
            }
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const int i = SIDES * m + side;
                float xa[8], xb[8], oa[8], ob[8];
                unpack8<T>(ra[m], xa);
                unpack8<T>(rb[m], xb);
                if (NORM && weight) {
                    float wa[8], wb[8];
                    unpack8<T>(weights[0], wa);
                    unpack8<T>(weights[1], wb);
                    const float r =
                        norm_factor<D>(sum_squares(xa) + sum_squares(xb), eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        xa[e] = xa[e] * r * wa[e];
                        xb[e] = xb[e] * r * wb[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float ce = c[e / 4][e % 4], se = s[e / 4][e % 4];
                    if constexpr (NORM) {
                        rotate_pair(xa[e], xb[e], ce, se, oa[e], ob[e]);
                    } else {
                        oa[e] = xa[e] * ce - xb[e] * se;
                        ob[e] = xb[e] * ce + xa[e] * se;
                    }
                }
                if (i < heads) {
                    store_chunk(j, i, c8, pack8<T>(oa));
                    store_chunk(j, i, c8 + CH / 2, pack8<T>(ob));
                }
            }
        }
    }

    // V: thread -> head dimension d = t, moved bit for bit
    if (V_APART ? v_only : !is_q)
        scatter_v_group<D, HB, (HB > 1)>(v_new + src_off, row_stride, g.count, heads, slot0, t,
                                         v_pages + tile);
}

// With norms, batches of one token a request: a group of rope_append_kernel leaves all but a token's lanes
// without work, so a wavefront of its own takes several heads of a token, 128 / (D/16) of keys or
// queries or 512 / D of V.  64 requests, 64/8 heads 3.0 us (4.4 in rope_append_kernel), 256 requests, 40/40
// heads 10.1 (13.9): 16 MB of rows, but a token's V is 2 of every 16 bytes of 21 MB.
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(64) void norm_rope_step_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in,
    uint16_t *q_out /* may be q_in */, const uint16_t *__restrict__ k_new,
    const uint16_t *__restrict__ v_new, const float *__restrict__ cos_sin,
    const int32_t *__restrict__ page_table, int32_t max_pages, int32_t num_q_heads,
    int32_t num_kv_heads, uint16_t *__restrict__ k_pages, uint16_t *__restrict__ v_pages,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps)
{
    typedef StepHeads<D> Heads;
    constexpr int VH = 512 / D;
    const AppendGroup g = groups[blockIdx.x];
    const int lane = lane_id();
    const int k_blocks = (num_kv_heads + Heads::kHeads - 1) / Heads::kHeads;
    const int v_blocks = (num_kv_heads + VH - 1) / VH;
    int y = (int)blockIdx.y;
    if (y >= k_blocks + v_blocks) {
        const Heads mine((y - k_blocks - v_blocks) * Heads::kHeads, num_q_heads);
        rotate_q<T, D, STYLE, 2, 1, false>(g, 0, 0, ((int64_t)g.q_row * num_q_heads + mine.first) * D,
                                           Heads::kEach * D, mine.count, q_in, q_out, q_weight, eps,
                                           cos_sin);
        return;
    }
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int slot = g.t_begin & 15;
    const int64_t row = (int64_t)g.q_row * num_kv_heads, tile = page * num_kv_heads;
    if (y < k_blocks) {
        const Heads mine(y * Heads::kHeads, num_kv_heads);
        const int c = lane % (D / 16);
        u32x4 rows[2][2], w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int h = mine.first + (i < mine.count ? i : 0) * Heads::kEach;
            rows[i][0] = load16(k_new + (row + h) * D + 8 * c);
            rows[i][1] = load16(k_new + (row + h) * D + D / 2 + 8 * c);
        }
        ChunkAngles<D, STYLE> angle;
        angle.load(cos_sin + (int64_t)g.t_begin * D, c);
        if (k_weight) {
            w[0] = load16(k_weight + 8 * c);
            w[1] = load16(k_weight + D / 2 + 8 * c);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            norm_rotate_chunks<T, D, STYLE>(rows[i], k_weight != nullptr, w, eps, angle);
            if (i < mine.count) {
                uint16_t *to = k_pages + (tile + mine.first + i * Heads::kEach) * (16 * D) + slot * 8;
                *reinterpret_cast<u32x4 *>(to + c * 128) = rows[i][0];
                *reinterpret_cast<u32x4 *>(to + (c + D / 16) * 128) = rows[i][1];
            }
        }
        return;
    }
    // V: lane -> head dimensions, moved bit for bit
    const int h0 = (y - k_blocks) * VH;
    uint16_t val[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = 64 * i + lane, h = min(h0 + at / D, num_kv_heads - 1);
        val[i] = v_new[(row + h) * D + at % D];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = 64 * i + lane, h = h0 + at / D;
        if (h < num_kv_heads)
            v_pages[(tile + h) * (16 * D) + ((slot >> 3) * D + at % D) * 8 + (slot & 7)] = val[i];
    }
}

template <typename T, int D, int STYLE>
static void launch_norm_step_t(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                               const void *k_new, const void *v_new, const int32_t *page_table,
                               void *k_pages, void *v_pages, hipStream_t stream)
{
    constexpr int KH = StepHeads<D>::kHeads, VH = 512 / D;
    const int hkv = plan->pool.num_kv_heads, hq = nr.q_in ? plan->num_q_heads : 0;
    const dim3 grid((unsigned)plan->append_groups.size(),
                    (unsigned)((hkv + KH - 1) / KH + (hkv + VH - 1) / VH + (hq + KH - 1) / KH));
    hipLaunchKernelGGL((norm_rope_step_kernel<T, D, STYLE>), grid, dim3(64), 0, stream,
                       dl.append_groups, (const uint16_t *)nr.q_in, (uint16_t *)nr.q_out,
                       (const uint16_t *)k_new, (const uint16_t *)v_new, nr.cos_sin,
                       page_table, plan->max_pages_per_req, plan->num_q_heads,
                       plan->pool.num_kv_heads, (uint16_t *)k_pages, (uint16_t *)v_pages,
                       (const uint16_t *)nr.q_weight, (const uint16_t *)nr.k_weight, nr.eps);
}

template <typename T, int D, int STYLE, int HB, bool NORM>
static void launch_rope_t(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                          const void *k_new, const void *v_new, const int32_t *page_table,
                          void *k_pages, void *v_pages, hipStream_t stream)
{
    const int kv_blocks = (plan->pool.num_kv_heads + HB - 1) / HB;
    const int q_blocks = nr.q_in ? (plan->num_q_heads + HB - 1) / HB : 0;
    const int v_blocks = kVApart<D, HB, NORM> ? kv_blocks : 0;
    const dim3 grid((unsigned)plan->append_groups.size(), (unsigned)(v_blocks + kv_blocks + q_blocks));
    hipLaunchKernelGGL((rope_append_kernel<T, D, STYLE, HB, NORM>), grid, dim3(D), 0, stream,
                       dl.append_groups, (const uint16_t *)nr.q_in, (uint16_t *)nr.q_out,
                       (const uint16_t *)k_new, (const uint16_t *)v_new, nr.cos_sin,
                       page_table, plan->max_pages_per_req, plan->num_q_heads,
                       plan->pool.num_kv_heads, (uint16_t *)k_pages, (uint16_t *)v_pages,
                       (const uint16_t *)nr.q_weight, (const uint16_t *)nr.k_weight, nr.eps);
}

// A large batch: two rows a thread (two heads a workgroup, four where pairs span the halves of a
// head and half of the threads do a head), and the rows are read with the streaming hint (kStreamBytes).
// 8 prompts, 7 K tokens, whole step: 40/40 heads, interleaved pairs 190 -> 181 us (187 with one head,
// 182 with four; 190 with four and no hint), half pairs 185 -> 177 (185 with two, 178 with eight);
// 64/8 heads, 4 K tokens, half pairs 95 -> 91.  A small batch keeps one head a workgroup, the more of
// them run at once (4 generation steps, 64/8 heads: 24.8 us against 25.5).
template <typename T, int D, bool NORM>
static auto pick_rope(int style, bool many, bool steps)
{
    if constexpr (NORM)
        if (steps) return style == 0 ? launch_norm_step_t<T, D, 0> : launch_norm_step_t<T, D, 1>;
    if (style == 0) return many ? launch_rope_t<T, D, 0, 2, NORM> : launch_rope_t<T, D, 0, 1, NORM>;
    return many ? launch_rope_t<T, D, 1, 4, NORM> : launch_rope_t<T, D, 1, 1, NORM>;
}

hipError_t launch_rope_append(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                              const void *k_new, const void *v_new, const int32_t *page_table,
                              void *k_pages, void *v_pages, hipStream_t stream)
{
    if (plan->append_groups.empty()) return hipSuccess;
    const bool f = plan->pool.dtype == PV_F16;
    const int64_t rows = 2 * plan->pool.num_kv_heads + (nr.q_in ? plan->num_q_heads : 0);
    const bool many = plan->total_q * rows * plan->pool.head_dim * 2 > kStreamBytes;
    const bool steps = (int32_t)plan->append_groups.size() == plan->total_q;  // one token a group
    auto pick = [&](auto norm) {
        constexpr bool NORM = decltype(norm)::value;
        return plan->pool.head_dim == 128
                   ? (f ? pick_rope<F16, 128, NORM>(nr.style, many, steps)
                        : pick_rope<BF16, 128, NORM>(nr.style, many, steps))
                   : (f ? pick_rope<F16, 64, NORM>(nr.style, many, steps)
                        : pick_rope<BF16, 64, NORM>(nr.style, many, steps));
    };
    auto go = nr.q_weight || nr.k_weight ? pick(std::true_type{}) : pick(std::false_type{});
    go(plan, dl, nr, k_new, v_new, page_table, k_pages, v_pages, stream);
    return hipGetLastError();
}

}  // namespace pv
