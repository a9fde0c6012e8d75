// The 8-bit pools: quantising K/V rows as they are appended (by themselves, or with the norm and the
// rotation of queries and keys in front), and reading rows back.
//
// What is computed (codes and scales: see pv_kv8.h).  For the new rows of one block (page, head; K
// and V apart) a = max |x| over their finite values, n = the least exponent with a <= 448 * 2^n.  In
// a page that is begun e = n; in one that holds earlier tokens e = max(its e, n), and where that is
// more than it was, the codes in front of the new ones are rounded anew for it.  Codes are x * 2^-e
// rounded to the nearest even; infinities and NaN become NaN.  Slots behind the new tokens keep
// their codes.
//
// Bound: HBM, and latency for generation steps.  One wavefront per block: a page's rows of one head
// are 4 KiB, 64 bytes a lane, so that the maximum over the block takes six lane exchanges and no LDS.
// K: lane = (slot, 16 dimensions of either half), whose codes are the pool's 16-byte chunks and
// which holds both partners of a rotation.  V: lane = two dimensions of all 16 slots, so that the
// transposition into the pool's runs of 16 slots is byte permutes inside a lane.
#include "pv_kv8.h"

namespace pv {

// Rows of the two 16-dimension chunks of a lane: dimensions 16c.. and D/2 + 16c..
template <int D>
__device__ __forceinline__ void load_halves(u32x4 (&raw)[4], const uint16_t *row, int c)
{
    raw[0] = load16(row + 16 * c);
    raw[1] = load16(row + 16 * c + 8);
    raw[2] = load16(row + D / 2 + 16 * c);
    raw[3] = load16(row + D / 2 + 16 * c + 8);
}

// y = x * w / sqrt(mean(x^2) + eps) (without a weight: y = x), rotated by the angles of the row's
// position; fp32 throughout, rounded to 16 bits once.  The D/32 lanes of a row are neighbours.
template <typename T, int D, int STYLE>
__device__ __forceinline__ void norm_rotate(u32x4 (&raw)[4], const uint16_t *weight, float eps,
                                            const float *cs, int c)
{
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack8<T>(raw[i], x[i]);
    if (weight) {  // the same for the whole workgroup
        const float r = norm_factor<D, 2>((sum_squares(x[0]) + sum_squares(x[2])) +
                                              (sum_squares(x[1]) + sum_squares(x[3])),
                                          eps);
        u32x4 wr[4];
        load_halves<D>(wr, weight, c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float w[8];
            unpack8<T>(wr[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * r * w[e];
        }
    }
    float y[4][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (STYLE == 1) {  // dimensions i and i + D/2
            const float *at = cs + 16 * c + 8 * i;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x4 co = *reinterpret_cast<const f32x4 *>(at + 4 * q);
                const f32x4 si = *reinterpret_cast<const f32x4 *>(at + D / 2 + 4 * q);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    rotate_pair(x[i][4 * q + e], x[i + 2][4 * q + e], co[e], si[e], y[i][4 * q + e],
                                y[i + 2][4 * q + e]);
            }
        } else {  // dimensions 2i and 2i + 1
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const float *at = cs + half * (D / 4) + 8 * c + 4 * i;
                const f32x4 co = *reinterpret_cast<const f32x4 *>(at);
                const f32x4 si = *reinterpret_cast<const f32x4 *>(at + D / 2);
                const int k = 2 * half + i;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    rotate_pair(x[k][2 * e], x[k][2 * e + 1], co[e], si[e], y[k][2 * e],
                                y[k][2 * e + 1]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = pack8<T>(y[i]);
}

// Exponent for the new rows of a block, whose magnitudes `mag` (a packed pair a lane) cover; the
// wavefront holds the whole block.  `before`: the page's exponent if it holds earlier tokens, else
// below every other.
template <typename T>
__device__ __forceinline__ int block_exponent(uint32_t mag, int before)
{
#pragma unroll
    for (int m = 32; m >= 1; m /= 2) mag = max_magnitudes(mag, __shfl_xor(mag, m));
    const uint32_t most = max(mag & 0xFFFFu, mag >> 16);
    return max(needed_exponent<T>(__builtin_amdgcn_readfirstlane((int)most)), before);
}
constexpr int kNoExponent = -1000;

// 16 values divided by the scale, as codes
template <typename T>
__device__ __forceinline__ u32x4 encode16(u32x4 a, u32x4 b, float scale)
{
    u32x4 codes;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const u32x4 &r = w < 2 ? a : b;
        const uint32_t lo = Kv8<T>::template encode2<false>(0u, r[2 * (w % 2)], scale);
        codes[w] = Kv8<T>::template encode2<true>(lo, r[2 * (w % 2) + 1], scale);
    }
    return codes;
}

// The codes of the slots in front of s0 in a K block, rounded anew by the whole wavefront
template <int D>
__device__ __forceinline__ void rescale_k(uint8_t *block, int s0, int before, int e)
{
    constexpr int LPT = D / 32;
    const int slot = lane_id() / LPT, c = lane_id() % LPT;
    if (slot >= s0) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        u32x4 *p = reinterpret_cast<u32x4 *>(block + kv8_k_chunk<D>(slot, c + half * LPT));
        u32x4 codes = *p;
#pragma unroll
        for (int w = 0; w < 4; ++w) codes[w] = rescale4(codes[w], before, e);
        *p = codes;
    }
}

template <typename T, int D, int STYLE>
__device__ __forceinline__ void append_k8(const AppendGroup &g, int h, int num_kv_heads, int64_t tile,
                                          const uint16_t *__restrict__ k_new,
                                          const uint16_t *weight, float eps, const float *cos_sin,
                                          uint8_t *__restrict__ k_pages, uint8_t *__restrict__ scales)
{
    constexpr int LPT = D / 32;  // lanes a token
    const int lane = lane_id();
    const int slot = lane / LPT, c = lane % LPT;
    const int s0 = g.t_begin & 15;
    const int j = min(max(slot - s0, 0), g.count - 1);
    const bool fresh = slot < 16 && slot >= s0 && slot < s0 + g.count;
    u32x4 raw[4];
    load_halves<D>(raw, k_new + ((int64_t)(g.q_row + j) * num_kv_heads + h) * D, c);
    const int before =
        s0 > 0 ? __builtin_amdgcn_readfirstlane((int)scales[tile]) - 127 : kNoExponent;
    if constexpr (STYLE >= 0)
        norm_rotate<T, D, STYLE>(raw, weight, eps, cos_sin + (int64_t)(g.t_begin + j) * D, c);
    uint32_t mag = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) mag = max_magnitudes(mag, finite_magnitudes<T>(raw[i][w]));
    const int e = block_exponent<T>(mag, before);
    if (e == Kv8<T>::kMaxExp) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) raw[i][w] = limit_to_top<T>(raw[i][w]);
    }
    const float scale = exp2_scale(e + 127);
    uint8_t *at = k_pages + tile * (16 * D);
    if (fresh) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
            *reinterpret_cast<u32x4 *>(at + kv8_k_chunk<D>(slot, c + half * LPT)) =
                encode16<T>(raw[2 * half], raw[2 * half + 1], scale);
    }
    if (s0 > 0 && e > before) rescale_k<D>(at, s0, before, e);
    if (lane == 0 && e != before) scales[tile] = (uint8_t)(e + 127);
}

template <typename T, int D>
__device__ __forceinline__ void append_v8(const AppendGroup &g, int h, int num_kv_heads, int64_t tile,
                                          const uint16_t *__restrict__ v_new,
                                          uint8_t *__restrict__ v_pages, uint8_t *__restrict__ scales)
{
    const int lane = lane_id();
    const int d = 2 * (lane % (D / 2));
    const int s0 = g.t_begin & 15, end = s0 + g.count;
    const uint16_t *src = v_new + ((int64_t)g.q_row * num_kv_heads + h) * D + d;
    uint32_t x[16];
#pragma unroll
    for (int s = 0; s < 16; ++s) {
        const int j = min(max(s - s0, 0), g.count - 1);
        x[s] = *reinterpret_cast<const uint32_t *>(src + (int64_t)j * num_kv_heads * D);
    }
    const int before =
        s0 > 0 ? __builtin_amdgcn_readfirstlane((int)scales[tile]) - 127 : kNoExponent;
    uint32_t mag = 0;
#pragma unroll
    for (int s = 0; s < 16; ++s) mag = max_magnitudes(mag, finite_magnitudes<T>(x[s]));
    const int e = block_exponent<T>(mag, before);
    if (e == Kv8<T>::kMaxExp) {
#pragma unroll
        for (int s = 0; s < 16; ++s) x[s] = limit_to_top<T>(x[s]);
    }
    const float scale = exp2_scale(e + 127);
    u32x4 codes[2];  // the 16 slots of dimensions d and d + 1
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t a = Kv8<T>::template encode2<false>(0u, x[4 * w], scale);
        a = Kv8<T>::template encode2<true>(a, x[4 * w + 1], scale);
        uint32_t b = Kv8<T>::template encode2<false>(0u, x[4 * w + 2], scale);
        b = Kv8<T>::template encode2<true>(b, x[4 * w + 3], scale);
        codes[0][w] = __builtin_amdgcn_perm(b, a, 0x06040200u);
        codes[1][w] = __builtin_amdgcn_perm(b, a, 0x07050301u);
    }
    uint8_t *at = v_pages + tile * (16 * D) + d * 16;
    if (lane < D / 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            u32x4 *p = reinterpret_cast<u32x4 *>(at + 16 * i);
            if (g.count < 16) {
                const u32x4 old = *p;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    // the bytes of word w in front of the new ones, and in front of their end
                    const uint32_t front = codes_in_front(s0 - 4 * w), upto = codes_in_front(end - 4 * w);
                    const uint32_t kept = s0 > 0 && e > before ? rescale4(old[w], before, e) : old[w];
                    codes[i][w] = (kept & front) | (codes[i][w] & upto & ~front) | (old[w] & ~upto);
                }
            }
            *p = codes[i];
        }
    }
    if (lane == 0 && e != before) scales[tile] = (uint8_t)(e + 127);
}

// Grid: (append groups, heads): the two wavefronts store K and V of a KV head, or, behind those,
// rotate the group's queries of two query heads.
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(128) void kv8_append_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in, uint16_t *q_out /* may be q_in */,
    const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps,
    const float *__restrict__ cos_sin, const int32_t *__restrict__ page_table, int32_t max_pages,
    int32_t num_q_heads, int32_t num_kv_heads, Kv8Ptrs pool)
{
    const AppendGroup g = groups[blockIdx.x];
    const int w = wave_id();
    int h = (int)blockIdx.y;
    if (STYLE >= 0 && h >= num_kv_heads) {
        constexpr int LPT = D / 32;
        h = 2 * (h - num_kv_heads) + w;
        const int j = lane_id() / LPT, c = lane_id() % LPT;
        if (h >= num_q_heads || j >= g.count) return;
        const int64_t row = ((int64_t)(g.q_row + j) * num_q_heads + h) * D;
        u32x4 raw[4];
        load_halves<D>(raw, q_in + row, c);
        norm_rotate<T, D, STYLE < 0 ? 0 : STYLE>(raw, q_weight, eps,
                                                 cos_sin + (int64_t)(g.t_begin + j) * D, c);
        uint16_t *to = q_out + row + 16 * c;
        *reinterpret_cast<u32x4 *>(to) = raw[0];
        *reinterpret_cast<u32x4 *>(to + 8) = raw[1];
        *reinterpret_cast<u32x4 *>(to + D / 2) = raw[2];
        *reinterpret_cast<u32x4 *>(to + D / 2 + 8) = raw[3];
        return;
    }
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int64_t tile = page * num_kv_heads + h;
    if (w == 0)
        append_k8<T, D, STYLE>(g, h, num_kv_heads, tile, k_new, k_weight, eps, cos_sin, pool.k,
                               pool.k_scales);
    else
        append_v8<T, D>(g, h, num_kv_heads, tile, v_new, pool.v, pool.v_scales);
}

// Batches that bring one token a request.  Whole pages a wavefront would leave most lanes without work,
// so a wavefront of its own takes several heads of one token: the K rows of 128 / (D / 16) heads (lane =
// head and the 32 dimensions of append_k8), V of a quarter as many (lane = 8 dimensions), or the
// queries of as many heads as K.  A page that has to be rounded anew is the whole wavefront's work.
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(64) void kv8_step_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in, uint16_t *q_out /* may be q_in */,
    const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps,
    const float *__restrict__ cos_sin, const int32_t *__restrict__ page_table, int32_t max_pages,
    int32_t num_q_heads, int32_t num_kv_heads, Kv8Ptrs pool)
{
    constexpr int LPT = D / 32, KH = 64 / LPT;  // lanes a head and heads, of K and queries
    constexpr int VL = D / 8, VH = 64 / VL;     // the same of V
    const AppendGroup g = groups[blockIdx.x];
    const int lane = lane_id();
    const int k_blocks = (num_kv_heads + KH - 1) / KH, v_blocks = (num_kv_heads + VH - 1) / VH;
    int y = (int)blockIdx.y;
    if (STYLE >= 0 && y >= k_blocks + v_blocks) {
        const int h = (y - k_blocks - v_blocks) * KH + lane / LPT, c = lane % LPT;
        if (h >= num_q_heads) return;
        const int64_t row = ((int64_t)g.q_row * num_q_heads + h) * D;
        u32x4 raw[4];
        load_halves<D>(raw, q_in + row, c);
        norm_rotate<T, D, STYLE < 0 ? 0 : STYLE>(raw, q_weight, eps, cos_sin + (int64_t)g.t_begin * D,
                                                 c);
        uint16_t *to = q_out + row + 16 * c;
        *reinterpret_cast<u32x4 *>(to) = raw[0];
        *reinterpret_cast<u32x4 *>(to + 8) = raw[1];
        *reinterpret_cast<u32x4 *>(to + D / 2) = raw[2];
        *reinterpret_cast<u32x4 *>(to + D / 2 + 8) = raw[3];
        return;
    }
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int s0 = g.t_begin & 15;
    if (y < k_blocks) {
        const int u = lane / LPT, c = lane % LPT;
        const bool valid = y * KH + u < num_kv_heads;
        const int h = valid ? y * KH + u : num_kv_heads - 1;
        const int64_t tile = page * num_kv_heads + h;
        u32x4 raw[4];
        load_halves<D>(raw, k_new + ((int64_t)g.q_row * num_kv_heads + h) * D, c);
        const int before = s0 > 0 ? (int)pool.k_scales[tile] - 127 : kNoExponent;
        if constexpr (STYLE >= 0)
            norm_rotate<T, D, STYLE>(raw, k_weight, eps, cos_sin + (int64_t)g.t_begin * D, c);
        uint32_t mag = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) mag = max_magnitudes(mag, finite_magnitudes<T>(raw[i][w]));
#pragma unroll
        for (int m = 1; m < LPT; m *= 2) mag = max_magnitudes(mag, __shfl_xor(mag, m));
        const int e = max(needed_exponent<T>(max(mag & 0xFFFFu, mag >> 16)), before);
        if (__any(e == Kv8<T>::kMaxExp)) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    raw[i][w] = e == Kv8<T>::kMaxExp ? limit_to_top<T>(raw[i][w]) : raw[i][w];
        }
        if (valid) {
            uint8_t *at = pool.k + tile * (16 * D);
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<u32x4 *>(at + kv8_k_chunk<D>(s0, c + half * LPT)) =
                    encode16<T>(raw[2 * half], raw[2 * half + 1], exp2_scale(e + 127));
            if (c == 0 && e != before) pool.k_scales[tile] = (uint8_t)(e + 127);
        }
        uint64_t grown = s0 > 0 ? __ballot(valid && c == 0 && e > before) : 0;
        for (; grown; grown &= grown - 1) {
            const int from = __ffsll((long long)grown) - 1;
            rescale_k<D>(pool.k + (page * num_kv_heads + y * KH + from / LPT) * (16 * D), s0,
                         __builtin_amdgcn_readlane(before, from), __builtin_amdgcn_readlane(e, from));
        }
        return;
    }
    y -= k_blocks;
    const int u = lane / VL, c = lane % VL;
    const bool valid = y * VH + u < num_kv_heads;
    const int h = valid ? y * VH + u : num_kv_heads - 1;
    const int64_t tile = page * num_kv_heads + h;
    u32x4 raw = load16(v_new + ((int64_t)g.q_row * num_kv_heads + h) * D + 8 * c);
    const int before = s0 > 0 ? (int)pool.v_scales[tile] - 127 : kNoExponent;
    uint32_t mag = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) mag = max_magnitudes(mag, finite_magnitudes<T>(raw[w]));
#pragma unroll
    for (int m = 1; m < VL; m *= 2) mag = max_magnitudes(mag, __shfl_xor(mag, m));
    const int e = max(needed_exponent<T>(max(mag & 0xFFFFu, mag >> 16)), before);
    if (__any(e == Kv8<T>::kMaxExp)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) raw[w] = e == Kv8<T>::kMaxExp ? limit_to_top<T>(raw[w]) : raw[w];
    }
    uint64_t grown = s0 > 0 ? __ballot(valid && c == 0 && e > before) : 0;
    if (grown) {
        for (; grown; grown &= grown - 1) {
            const int from = __ffsll((long long)grown) - 1;
            const int b = __builtin_amdgcn_readlane(before, from);
            const int a = __builtin_amdgcn_readlane(e, from);
            uint8_t *at = pool.v + (page * num_kv_heads + y * VH + from / VL) * (16 * D);
            for (int d = lane; d < D; d += 64) {
                u32x4 *p = reinterpret_cast<u32x4 *>(at + d * 16);
                u32x4 codes = *p;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t front = codes_in_front(s0 - 4 * w);
                    codes[w] = (rescale4(codes[w], b, a) & front) | (codes[w] & ~front);
                }
                *p = codes;
            }
        }
        __builtin_amdgcn_s_waitcnt(0);  // the new token's codes, below, lie among these bytes
        asm volatile("" ::: "memory");
    }
    if (valid) {
        uint8_t *at = pool.v + tile * (16 * D) + c * 128 + s0;
        const float scale = exp2_scale(e + 127);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t two = Kv8<T>::template encode2<false>(0u, raw[w], scale);
            at[32 * w] = (uint8_t)two;
            at[32 * w + 16] = (uint8_t)(two >> 8);
        }
        if (c == 0 && e != before) pool.v_scales[tile] = (uint8_t)(e + 127);
    }
}

// The inverse: the rows of the plan's new tokens out of the pools, as 16-bit values (exact).
template <typename T, int D>
__global__ __launch_bounds__(128) void kv8_read_kernel(
    const AppendGroup *__restrict__ groups, Kv8Ptrs pool, const int32_t *__restrict__ page_table,
    int32_t max_pages, int32_t num_kv_heads, uint16_t *__restrict__ k_rows,
    uint16_t *__restrict__ v_rows)
{
    const AppendGroup g = groups[blockIdx.x];
    const int h = (int)blockIdx.y;
    const int lane = lane_id();
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int64_t tile = page * num_kv_heads + h;
    const int s0 = g.t_begin & 15;
    const int64_t stride = (int64_t)num_kv_heads * D;
    const int64_t first = (int64_t)g.q_row * stride + (int64_t)h * D;
    if (wave_id() == 0) {
        constexpr int LPT = D / 32;
        const float scale = exp2_scale(pool.k_scales[tile]);
        const int slot = lane / LPT, c = lane % LPT;
        if (slot < s0 || slot >= s0 + g.count) return;
        uint16_t *to = k_rows + first + (slot - s0) * stride;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int chunk = c + half * LPT;
            const u32x4 codes = load16(pool.k + tile * (16 * D) + kv8_k_chunk<D>(slot, chunk));
            *reinterpret_cast<u32x4 *>(to + 16 * chunk) = decode8<T>(codes[0], codes[1], scale);
            *reinterpret_cast<u32x4 *>(to + 16 * chunk + 8) = decode8<T>(codes[2], codes[3], scale);
        }
    } else {
        if (lane >= D / 2) return;
        const float scale = exp2_scale(pool.v_scales[tile]);
        const int d = 2 * lane;
        const uint8_t *from = pool.v + tile * (16 * D) + d * 16;
        const u32x4 a = load16(from), b = load16(from + 16);
        uint16_t *to = v_rows + first + d;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t a0 = Kv8<T>::template decode2<false>(a[w], scale);
            const uint32_t a1 = Kv8<T>::template decode2<true>(a[w], scale);
            const uint32_t b0 = Kv8<T>::template decode2<false>(b[w], scale);
            const uint32_t b1 = Kv8<T>::template decode2<true>(b[w], scale);
            const uint32_t row[4] = {
                __builtin_amdgcn_perm(b0, a0, 0x05040100u), __builtin_amdgcn_perm(b0, a0, 0x07060302u),
                __builtin_amdgcn_perm(b1, a1, 0x05040100u), __builtin_amdgcn_perm(b1, a1, 0x07060302u)};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int slot = 4 * w + i;
                if (slot >= s0 && slot < s0 + g.count)
                    *reinterpret_cast<uint32_t *>(to + (slot - s0) * stride) = row[i];
            }
        }
    }
}

template <typename T, int D, int STYLE>
static void launch_append8_t(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                             const void *k_new, const void *v_new, const int32_t *page_table,
                             const Kv8Ptrs &pool, hipStream_t stream)
{
    const int hq = STYLE >= 0 && nr.q_in ? plan->num_q_heads : 0, hkv = plan->pool.num_kv_heads;
    const bool steps = (int32_t)plan->append_groups.size() == plan->total_q;  // one token a group
    constexpr int KH = 64 / (D / 32), VH = 64 / (D / 8);
    const int blocks = steps ? (hkv + KH - 1) / KH + (hkv + VH - 1) / VH + (hq + KH - 1) / KH
                             : hkv + (hq + 1) / 2;
    const dim3 grid((unsigned)plan->append_groups.size(), (unsigned)blocks);
    auto kernel = steps ? kv8_step_kernel<T, D, STYLE> : kv8_append_kernel<T, D, STYLE>;
    hipLaunchKernelGGL(kernel, grid, dim3(steps ? 64 : 128), 0, stream,
                       dl.append_groups, (const uint16_t *)nr.q_in, (uint16_t *)nr.q_out,
                       (const uint16_t *)k_new, (const uint16_t *)v_new,
                       (const uint16_t *)nr.q_weight, (const uint16_t *)nr.k_weight, nr.eps,
                       nr.cos_sin, page_table, plan->max_pages_per_req, plan->num_q_heads,
                       plan->pool.num_kv_heads, pool);
}

template <typename T, int D>
static auto pick_append8(int style)
{
    return style < 0    ? launch_append8_t<T, D, -1>
           : style == 0 ? launch_append8_t<T, D, 0>
                        : launch_append8_t<T, D, 1>;
}

hipError_t launch_kv8_append(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                             const void *k_new, const void *v_new, const int32_t *page_table,
                             const pv_kv8_pool &pool, hipStream_t stream)
{
    if (plan->append_groups.empty()) return hipSuccess;
    const bool f = plan->pool.dtype == PV_F16;
    auto go = plan->pool.head_dim == 128
                  ? (f ? pick_append8<F16, 128>(nr.style) : pick_append8<BF16, 128>(nr.style))
                  : (f ? pick_append8<F16, 64>(nr.style) : pick_append8<BF16, 64>(nr.style));
    const Kv8Ptrs p = {static_cast<uint8_t *>(pool.k), static_cast<uint8_t *>(pool.v), pool.k_scales,
                       pool.v_scales};
    go(plan, dl, nr, k_new, v_new, page_table, p, stream);
    return hipGetLastError();
}

hipError_t launch_kv8_read(const pv_plan *plan, const DeviceLists &dl, const pv_kv8_pool &pool,
                           const int32_t *page_table, void *k_rows, void *v_rows,
                           hipStream_t stream)
{
    if (plan->append_groups.empty()) return hipSuccess;
    const bool f = plan->pool.dtype == PV_F16;
    const Kv8Ptrs p = {static_cast<uint8_t *>(pool.k), static_cast<uint8_t *>(pool.v), pool.k_scales,
                       pool.v_scales};
    auto kernel = plan->pool.head_dim == 128 ? (f ? kv8_read_kernel<F16, 128> : kv8_read_kernel<BF16, 128>)
                                             : (f ? kv8_read_kernel<F16, 64> : kv8_read_kernel<BF16, 64>);
    const dim3 grid((unsigned)plan->append_groups.size(), (unsigned)plan->pool.num_kv_heads);
    hipLaunchKernelGGL(kernel, grid, dim3(128), 0, stream, dl.append_groups, p, page_table,
                       plan->max_pages_per_req, plan->pool.num_kv_heads, (uint16_t *)k_rows,
                       (uint16_t *)v_rows);
    return hipGetLastError();
}

}  // namespace pv
