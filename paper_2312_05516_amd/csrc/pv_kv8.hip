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
// transposition into the pool's runs of 16 slots is byte permutes inside a lane.  Queries, which are not
// quantised: D/16 lanes a row, 16 bytes of either half side by side (32 bytes a lane, as K has them: 40.0 us
// for 4.4 K tokens, 64/8 heads, 38.4 so).
//
// Measured: 8 prompts, 6.5 K tokens, 40 KV heads, 201 MB in 38.2 us = 5.25 TB/s (a device copy of 1 GiB:
// 5.2); reading 70 K tokens of 8 heads back, 427 MB in 85.1 us = 5.0 TB/s; norms and rotation in front, 4.4 K
// tokens, 64/8 heads, 172 MB in 33.7 us = 5.1 TB/s; 256 generation steps 3.6 us, launch and latency.
#include "pv_kv8.h"
#include "pv_norm_rope.h"

namespace pv {

// Rows of the two 16-dimension chunks of a lane: dimensions 16c.. and D/2 + 16c..
template <int D, bool STREAM>
__device__ __forceinline__ void load_halves(u32x4 (&raw)[4], const uint16_t *row, int c)
{
    raw[0] = load16_as<STREAM>(row + 16 * c);
    raw[1] = load16_as<STREAM>(row + 16 * c + 8);
    raw[2] = load16_as<STREAM>(row + D / 2 + 16 * c);
    raw[3] = load16_as<STREAM>(row + D / 2 + 16 * c + 8);
}

// Cosines and sines of a lane's pairs: of dimensions 16c + i and D/2 + 16c + i (STYLE 1), or of the
// neighbours in both chunks (STYLE 0).  The heads of a token share them.
template <int D, int STYLE>
struct Angles {
    f32x4 c[4], s[4];
    __device__ __forceinline__ void load(const float *cs, int lane_c)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float *at =
                cs + (STYLE == 1 ? 16 * lane_c + 4 * k : k / 2 * (D / 4) + 8 * lane_c + k % 2 * 4);
            c[k] = *reinterpret_cast<const f32x4 *>(at);
            s[k] = *reinterpret_cast<const f32x4 *>(at + D / 2);
        }
    }
};

// y = x * w / sqrt(mean(x^2) + eps) (without a weight: y = x), rotated by the angles of the row's
// position; fp32 throughout, rounded to 16 bits once.  The D/32 lanes of a row are neighbours.
template <typename T, int D, int STYLE>
__device__ __forceinline__ void norm_rotate(u32x4 (&raw)[4], bool norm, const u32x4 (&weight)[4],
                                            float eps, const Angles<D, STYLE> &angle)
{
    float x[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack8<T>(raw[i], x[i]);
    if (norm) {  // the same for the whole workgroup
        const float r = norm_factor<D, 2>((sum_squares(x[0]) + sum_squares(x[2])) +
                                              (sum_squares(x[1]) + sum_squares(x[3])),
                                          eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float w[8];
            unpack8<T>(weight[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * r * w[e];
        }
    }
    float y[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (STYLE == 1) {  // dimensions i and i + D/2
                const int i = k / 2, at = 4 * (k % 2) + e;
                rotate_pair(x[i][at], x[i + 2][at], angle.c[k][e], angle.s[k][e], y[i][at],
                            y[i + 2][at]);
            } else {  // dimensions 2i and 2i + 1
                rotate_pair(x[k][2 * e], x[k][2 * e + 1], angle.c[k][e], angle.s[k][e], y[k][2 * e],
                            y[k][2 * e + 1]);
            }
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = pack8<T>(y[i]);
}

// A wavefront works on one block of head size 128, or on two of head size 64 side by side, the second
// with its upper lanes.
template <int D>
struct Side {
    static constexpr int kHeads = 128 / D, kLanes = 64 / kHeads;
    // head of the lane (0 or 1), and the lane's place in its block's lanes
    static __device__ __forceinline__ int head() { return D == 128 ? 0 : lane_id() / kLanes; }
    static __device__ __forceinline__ int lane() { return lane_id() % kLanes; }
};

// Exponent for the new rows of a block, whose magnitudes `mag` (a packed pair a lane) cover.  `before`:
// the page's exponent if it holds earlier tokens, else below every other.
template <typename T, int D>
__device__ __forceinline__ int block_exponent(uint32_t mag, int before)
{
    mag = max_of_lanes<Side<D>::kLanes>(mag);
    int most = (int)max(mag & 0xFFFFu, mag >> 16);
    if (D == 128) most = __builtin_amdgcn_readfirstlane(most);
    return max(needed_exponent<T>((uint32_t)most), before);
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

// The codes of the slots in front of s0 in a K block, rounded anew by all of its lanes, `at` being
// the lane's place among them
template <int D>
__device__ __forceinline__ void rescale_k(uint8_t *block, int at, int s0, int before, int e)
{
    constexpr int LPT = D / 32;
    const int slot = at / LPT, c = at % LPT;
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

// K of HB * Side<D>::kHeads heads of a page, of which `heads` exist; `tile` is the first one's block.
// All rows are loaded before the first is worked on.
template <typename T, int D, int STYLE, int HB, bool STREAM>
__device__ __forceinline__ void append_k8(const AppendGroup &g, int h, int heads, int num_kv_heads,
                                          int64_t tile, const uint16_t *__restrict__ k_new,
                                          const uint16_t *weight, float eps, const float *cos_sin,
                                          uint8_t *__restrict__ k_pages, uint8_t *__restrict__ scales)
{
    constexpr int LPT = D / 32;  // lanes a token
    constexpr int SH = Side<D>::kHeads;
    const int lane = Side<D>::lane(), side = Side<D>::head();
    const int slot = lane / LPT, c = lane % LPT;
    const int s0 = g.t_begin & 15;
    const int j = min(max(slot - s0, 0), g.count - 1);
    const bool fresh = slot >= s0 && slot < s0 + g.count;
    u32x4 rows[HB][4];
    int before[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        const int at = i * SH + side < heads ? i * SH + side : 0;
        load_halves<D, STREAM>(rows[i], k_new + ((int64_t)(g.q_row + j) * num_kv_heads + h + at) * D, c);
        before[i] = s0 > 0 ? (int)scales[tile + at] - 127 : kNoExponent;
        if (D == 128) before[i] = __builtin_amdgcn_readfirstlane(before[i]);
    }
    Angles<D, STYLE < 0 ? 0 : STYLE> angle;
    u32x4 w[4];
    if constexpr (STYLE >= 0) {
        angle.load(cos_sin + (int64_t)(g.t_begin + j) * D, c);
        if (weight) load_halves<D, false>(w, weight, c);
    }
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i * SH >= heads) break;
        const int at_head = i * SH + side;
        const bool valid = SH == 1 || at_head < heads;
        u32x4 (&raw)[4] = rows[i];
        if constexpr (STYLE >= 0) norm_rotate<T, D, STYLE>(raw, weight != nullptr, w, eps, angle);
        uint32_t mag = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int q = 0; q < 4; ++q) mag = max_magnitudes(mag, finite_magnitudes<T>(raw[k][q]));
        const int e = block_exponent<T, D>(mag, before[i]);
        if (e == Kv8<T>::kMaxExp) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) raw[k][q] = limit_to_top<T>(raw[k][q]);
        }
        const float scale = exp2_scale(e + 127);
        uint8_t *at = k_pages + (tile + at_head) * (16 * D);
        if (fresh && valid) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
                *reinterpret_cast<u32x4 *>(at + kv8_k_chunk<D>(slot, c + half * LPT)) =
                    encode16<T>(raw[2 * half], raw[2 * half + 1], scale);
        }
        if (s0 > 0 && e > before[i] && valid) rescale_k<D>(at, lane, s0, before[i], e);
        if (lane == 0 && e != before[i] && valid) scales[tile + at_head] = (uint8_t)(e + 127);
    }
}

template <typename T, int D, int HB, bool STREAM>
__device__ __forceinline__ void append_v8(const AppendGroup &g, int h, int heads, int num_kv_heads,
                                          int64_t tile, const uint16_t *__restrict__ v_new,
                                          uint8_t *__restrict__ v_pages, uint8_t *__restrict__ scales)
{
    constexpr int SH = Side<D>::kHeads;
    const int lane = Side<D>::lane(), side = Side<D>::head();
    const int d = 2 * lane;
    const int s0 = g.t_begin & 15, end = s0 + g.count;
    const uint16_t *src = v_new + ((int64_t)g.q_row * num_kv_heads + h) * D + d;
    uint32_t rows[HB][16];
    int exps[HB];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        const int at = i * SH + side < heads ? i * SH + side : 0;
#pragma unroll
        for (int s = 0; s < 16; ++s) {
            const int j = min(max(s - s0, 0), g.count - 1);
            const uint32_t *from =
                reinterpret_cast<const uint32_t *>(src + ((int64_t)j * num_kv_heads + at) * D);
            rows[i][s] = STREAM ? __builtin_nontemporal_load(from) : *from;
        }
        exps[i] = s0 > 0 ? (int)scales[tile + at] - 127 : kNoExponent;
        if (D == 128) exps[i] = __builtin_amdgcn_readfirstlane(exps[i]);
    }
#pragma unroll
    for (int i = 0; i < HB; ++i) {
        if (i * SH >= heads) break;
        const int at_head = i * SH + side;
        const bool valid = SH == 1 || at_head < heads;
        uint32_t (&x)[16] = rows[i];
        const int before = exps[i];
        uint32_t mag = 0;
#pragma unroll
        for (int s = 0; s < 16; ++s) mag = max_magnitudes(mag, finite_magnitudes<T>(x[s]));
        const int e = block_exponent<T, D>(mag, before);
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
        if (valid) {
            uint8_t *at = v_pages + (tile + at_head) * (16 * D) + d * 16;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                u32x4 *p = reinterpret_cast<u32x4 *>(at + 16 * k);
                if (g.count < 16) {
                    const u32x4 old = *p;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        // the bytes of word w in front of the new ones, and in front of their end
                        const uint32_t front = codes_in_front(s0 - 4 * w);
                        const uint32_t upto = codes_in_front(end - 4 * w);
                        const uint32_t kept = s0 > 0 && e > before ? rescale4(old[w], before, e) : old[w];
                        codes[k][w] = (kept & front) | (codes[k][w] & upto & ~front) | (old[w] & ~upto);
                    }
                }
                *p = codes[k];
            }
        }
        if (lane == 0 && e != before && valid) scales[tile + at_head] = (uint8_t)(e + 127);
    }
}

// Grid: (append groups, blocks of heads): the two wavefronts store K and V of HB KV heads (twice as
// many of head size 64), or, behind those, rotate the queries of as many query heads each.
template <typename T, int D, int STYLE, int HB, bool STREAM>
__global__ __launch_bounds__(128) void kv8_append_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in, uint16_t *q_out /* may be q_in */,
    const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps,
    const float *__restrict__ cos_sin, const int32_t *__restrict__ page_table, int32_t max_pages,
    int32_t num_q_heads, int32_t num_kv_heads, Kv8Ptrs pool)
{
    constexpr int SH = Side<D>::kHeads, HEADS = HB * SH;
    const AppendGroup g = groups[blockIdx.x];
    const int w = wave_id();
    const int kv_blocks = (num_kv_heads + HEADS - 1) / HEADS;
    if (STYLE >= 0 && (int)blockIdx.y >= kv_blocks) {
        const int h = (2 * ((int)blockIdx.y - kv_blocks) + w) * HEADS;
        if (h >= num_q_heads) return;
        rotate_q<T, D, STYLE < 0 ? 0 : STYLE, HEADS, D / 64, STREAM>(
            g, lane_id() / (D / 16), (int64_t)num_q_heads * D,
            ((int64_t)g.q_row * num_q_heads + h) * D, D, num_q_heads - h, q_in, q_out, q_weight, eps,
            cos_sin);
        return;
    }
    const int h = (int)blockIdx.y * HEADS, heads = min(HEADS, num_kv_heads - h);
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int64_t tile = page * num_kv_heads + h;
    if (w == 0)
        append_k8<T, D, STYLE, HB, STREAM>(g, h, heads, num_kv_heads, tile, k_new, k_weight, eps,
                                           cos_sin, pool.k, pool.k_scales);
    else
        append_v8<T, D, HB, STREAM>(g, h, heads, num_kv_heads, tile, v_new, pool.v, pool.v_scales);
}

// Batches that bring one token a request.  Whole pages a wavefront would leave most lanes without work,
// so a wavefront of its own takes several heads of one token: the K rows of 128 / (D / 16) heads (lane =
// head and the 32 dimensions of append_k8), V of two, or the queries of as many heads as K.  A page that has
// to be rounded anew is the whole wavefront's work.  V's codes lie 16 bytes apart, a line for eight of them:
// with neighbouring lanes on neighbouring dimensions 256 requests, 40 heads take 8.6 us (12.2 with 8
// dimensions a lane), 8 heads 3.6 (4.4); four heads of V a wavefront 8.5 and 3.75, 32 requests 2.83 (2.66).
constexpr int kStepHeadsV = 2;
template <typename T, int D, int STYLE>
__global__ __launch_bounds__(64) void kv8_step_kernel(
    const AppendGroup *__restrict__ groups, const uint16_t *q_in, uint16_t *q_out /* may be q_in */,
    const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
    const uint16_t *__restrict__ q_weight, const uint16_t *__restrict__ k_weight, float eps,
    const float *__restrict__ cos_sin, const int32_t *__restrict__ page_table, int32_t max_pages,
    int32_t num_q_heads, int32_t num_kv_heads, Kv8Ptrs pool)
{
    constexpr int LPT = D / 32, KH = 64 / LPT;  // lanes a head and heads, of K and queries
    constexpr int VH = kStepHeadsV;             // heads of V
    const AppendGroup g = groups[blockIdx.x];
    const int lane = lane_id();
    const int k_blocks = (num_kv_heads + KH - 1) / KH, v_blocks = (num_kv_heads + VH - 1) / VH;
    int y = (int)blockIdx.y;
    if (STYLE >= 0 && y >= k_blocks + v_blocks) {
        static_assert(StepHeads<D>::kHeads == KH, "queries go in as many blocks as keys");
        const StepHeads<D> mine((y - k_blocks - v_blocks) * KH, num_q_heads);
        rotate_q<T, D, STYLE < 0 ? 0 : STYLE, 2, 1, false>(
            g, 0, 0, ((int64_t)g.q_row * num_q_heads + mine.first) * D, StepHeads<D>::kEach * D,
            mine.count, q_in, q_out, q_weight, eps, cos_sin);
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
        load_halves<D, false>(raw, k_new + ((int64_t)g.q_row * num_kv_heads + h) * D, c);
        const int before = s0 > 0 ? (int)pool.k_scales[tile] - 127 : kNoExponent;
        if constexpr (STYLE >= 0) {
            Angles<D, STYLE> angle;
            angle.load(cos_sin + (int64_t)g.t_begin * D, c);
            u32x4 w[4];
            if (k_weight) load_halves<D, false>(w, k_weight, c);
            norm_rotate<T, D, STYLE>(raw, k_weight != nullptr, w, eps, angle);
        }
        uint32_t mag = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) mag = max_magnitudes(mag, finite_magnitudes<T>(raw[i][w]));
        mag = max_of_lanes<LPT>(mag);
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
            rescale_k<D>(pool.k + (page * num_kv_heads + y * KH + from / LPT) * (16 * D), lane, s0,
                         __builtin_amdgcn_readlane(before, from), __builtin_amdgcn_readlane(e, from));
        }
        return;
    }
    y -= k_blocks;
    // V: a lane holds dimensions lane, lane + 64, .. of the heads one behind the other, so that its codes lie
    // 16 bytes from its neighbours'.  values[i / 2] holds the i-th; the heads' exponents are the wavefront's.
    const int h0 = y * VH, heads = min(VH, num_kv_heads - h0);
    constexpr int EACH = D / 64, N = VH * EACH;  // values of a head, and of all
    const int64_t tile = page * num_kv_heads + h0;
    const int scales = pool.v_scales[tile + min(lane, heads - 1)];  // of a page that is begun: not used
    uint32_t values[N / 2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int h = h0 + (i / EACH < heads ? i / EACH : 0);
        const uint32_t x = v_new[((int64_t)g.q_row * num_kv_heads + h) * D + i % EACH * 64 + lane];
        values[i / 2] = i % 2 ? values[i / 2] | x << 16 : x;
    }
    int before[VH], e[VH];
#pragma unroll
    for (int i = 0; i < VH; ++i)
        before[i] = s0 > 0 ? __builtin_amdgcn_readlane(scales, i) - 127 : kNoExponent;
    uint32_t mags[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) mags[i] = finite_magnitudes<T>(values[i]);
#pragma unroll
    for (int i = 0; i < VH; i += 2) {  // two heads' magnitudes side by side
        uint32_t two = mags[i / 2];  // EACH == 1: values hold them so
        if constexpr (EACH == 2) {
            const uint32_t a = mags[i], b = mags[i + 1];
            two = (max_magnitudes(a, a >> 16) & 0xFFFFu) | (max_magnitudes(b, b << 16) & 0xFFFF0000u);
        }
        two = __builtin_amdgcn_readfirstlane(max_of_lanes<64>(two));
        e[i] = max(needed_exponent<T>(two & 0xFFFFu), before[i]);
        e[i + 1] = max(needed_exponent<T>(two >> 16), before[i + 1]);
    }
    bool grown = false;
#pragma unroll
    for (int i = 0; i < VH; ++i) grown |= i < heads && s0 > 0 && e[i] > before[i];
    if (grown) {
#pragma unroll 1
        for (int i = 0; i < heads; ++i) {
            const int from = __builtin_amdgcn_readlane(scales, i) - 127;
            int to = e[0];
#pragma unroll
            for (int k = 1; k < VH; ++k) to = i == k ? e[k] : to;
            if (to <= from) continue;
            for (int d = lane; d < D; d += 64) {
                u32x4 *p = reinterpret_cast<u32x4 *>(pool.v + (tile + i) * (16 * D) + d * 16);
                u32x4 codes = *p;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t front = codes_in_front(s0 - 4 * w);
                    codes[w] = (rescale4(codes[w], from, to) & front) | (codes[w] & ~front);
                }
                *p = codes;
            }
        }
        __builtin_amdgcn_s_waitcnt(0);  // the new token's codes, below, lie among these bytes
        asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < VH; ++i) {
        if (i >= heads) break;
        const float scale = exp2_scale(e[i] + 127);
        uint32_t xy = EACH == 2 ? values[i] : i % 2 ? values[i / 2] >> 16 : values[i / 2] & 0xFFFFu;
        if (e[i] == Kv8<T>::kMaxExp) xy = limit_to_top<T>(xy);
        const uint32_t codes = Kv8<T>::template encode2<false>(0u, xy, scale);
        uint8_t *at = pool.v + (tile + i) * (16 * D) + lane * 16 + s0;
        at[0] = (uint8_t)codes;
        if constexpr (EACH == 2) at[64 * 16] = (uint8_t)(codes >> 8);
        if (lane == 0 && e[i] != before[i]) pool.v_scales[tile + i] = (uint8_t)(e[i] + 127);
    }
}

// The inverse: the rows of the plan's new tokens out of the pools, as 16-bit values (exact).  One
// wavefront reads K, one V, of HB heads of a page, all their codes before the first is converted.  K:
// lane = 8 dimensions of a slot, so that a store is whole rows.  V: lane = 4 dimensions of 8 slots, so
// that half a wavefront stores a row.
template <typename T, int D, int HB>
__global__ __launch_bounds__(128) void kv8_read_kernel(
    const AppendGroup *__restrict__ groups, Kv8Ptrs pool, const int32_t *__restrict__ page_table,
    int32_t max_pages, int32_t num_kv_heads, uint16_t *__restrict__ k_rows,
    uint16_t *__restrict__ v_rows)
{
    const AppendGroup g = groups[blockIdx.x];
    const int h0 = (int)blockIdx.y * HB, heads = min(HB, num_kv_heads - h0);
    const int lane = lane_id();
    const int64_t page = page_table[(int64_t)g.req * max_pages + (g.t_begin >> 4)];
    const int64_t tile = page * num_kv_heads + h0;
    const int s0 = g.t_begin & 15;
    const int64_t stride = (int64_t)num_kv_heads * D;
    const int64_t first = (int64_t)g.q_row * stride + (int64_t)h0 * D;
    if (wave_id() == 0) {
        constexpr int LPR = D / 8, STEPS = 16 * LPR / 64;  // lanes a row; rows of 64 lanes
        const int c = lane % LPR;
        u32x2 codes[HB][STEPS];
        uint32_t e[HB];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int64_t t = tile + (i < heads ? i : 0);
            e[i] = pool.k_scales[t];
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
                codes[i][k] = *reinterpret_cast<const u32x2 *>(
                    pool.k + t * (16 * D) + kv8_k_chunk<D>(64 / LPR * k + lane / LPR, c / 2) + c % 2 * 8);
        }
#pragma unroll
        for (int i = 0; i < HB; ++i)
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const int j = 64 / LPR * k + lane / LPR - s0;
                if (i < heads && j >= 0 && j < g.count)
                    *reinterpret_cast<u32x4 *>(k_rows + first + j * stride + i * D + 8 * c) =
                        decode8<T>(codes[i][k][0], codes[i][k][1], exp2_scale((int)e[i]));
            }
    } else {
        constexpr int ROWS = 256 / D;  // rows of 4 dimensions a lane in a wavefront: 2, or 4
        constexpr int PER = 16 / ROWS; // consecutive slots of a lane: 8, or 4
        const int d = 4 * (lane % (D / 4)), part = lane / (D / 4);
        uint32_t codes[HB][4][PER / 4];
        uint32_t e[HB];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const int64_t t = tile + (i < heads ? i : 0);
            e[i] = pool.v_scales[t];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint8_t *from = pool.v + t * (16 * D) + (d + k) * 16 + part * PER;
                if constexpr (PER == 8) {
                    const u32x2 v = *reinterpret_cast<const u32x2 *>(from);
                    codes[i][k][0] = v[0];
                    codes[i][k][PER / 4 - 1] = v[1];
                } else {
                    codes[i][k][0] = *reinterpret_cast<const uint32_t *>(from);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const float scale = exp2_scale((int)e[i]);
#pragma unroll
            for (int w = 0; w < PER / 4; ++w) {
                uint32_t lo[4], hi[4];  // slots 0, 1 and 2, 3 of the four dimensions
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    lo[k] = Kv8<T>::template decode2<false>(codes[i][k][w], scale);
                    hi[k] = Kv8<T>::template decode2<true>(codes[i][k][w], scale);
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const uint32_t *x = s < 2 ? lo : hi;
                    const uint32_t pick = s % 2 ? 0x07060302u : 0x05040100u;
                    const int j = part * PER + 4 * w + s - s0;
                    if (i < heads && j >= 0 && j < g.count)
                        *reinterpret_cast<u32x2 *>(v_rows + first + j * stride + i * D + d) =
                            u32x2{__builtin_amdgcn_perm(x[1], x[0], pick),
                                  __builtin_amdgcn_perm(x[3], x[2], pick)};
                }
            }
        }
    }
}

// Rules, us a call (three batches in turn, so that small ones find their rows in a cache):
//  * Batches of one token a request take the kernel for them: 256 requests, 8 KV heads 3.6 (5.5 with the
//    kernel for pages), 40 heads 8.6 (15.7).
//  * With rotation more than 32 MiB of rows take two heads a wavefront, which share the angles: 6
//    prompts, 40/40 heads, 4.8 K tokens 53.3 (one: 56.0), 8 of 300, 64/8 heads 21.1 (22.8), but 2 of 100
//    5.6 (4.3).  Without rotation one head is ahead (6 K tokens, 40 heads: 39.7, two 41.4).
//  * More than 64 MiB of rows, with rotation more than 48 and head size 128, are read with the streaming
//    hint.  Without rotation 6 K tokens, 40 heads 36.0 (39.7 without the hint), 4 K 25.3 (26.9), 3 K 24.3
//    (22.3).  With it 4.4 K tokens, 64/8 heads 33.7 (38.4), 3.2 K 25.9 (29.0), 2.4 K 21.1 (21.2); 4.8 K, 40/40
//    heads 50.0 (53.3).  Head size 64, whose half rows are half a cache line: 22 K tokens, 32/8 heads 59.4
//    (56.8).
template <typename T, int D, int STYLE>
static void launch_append8_t(const pv_plan *plan, const DeviceLists &dl, const NormRope &nr,
                             const void *k_new, const void *v_new, const int32_t *page_table,
                             const Kv8Ptrs &pool, hipStream_t stream)
{
    const int hq = STYLE >= 0 && nr.q_in ? plan->num_q_heads : 0, hkv = plan->pool.num_kv_heads;
    const int64_t row_bytes = (int64_t)plan->total_q * (2 * hkv + hq) * D * 2;
    const bool steps = (int32_t)plan->append_groups.size() == plan->total_q;  // one token a group
    const bool two = STYLE >= 0 && row_bytes > kStreamBytes;
    const bool streams = STYLE < 0 ? row_bytes > 2 * kStreamBytes
                                   : D == 128 && 2 * row_bytes > 3 * kStreamBytes;
    constexpr int KH = 64 / (D / 32), VH = kStepHeadsV;
    const int heads = (two ? 2 : 1) * (128 / D);
    const int blocks = steps ? (hkv + KH - 1) / KH + (hkv + VH - 1) / VH + (hq + KH - 1) / KH
                             : (hkv + heads - 1) / heads + (hq + 2 * heads - 1) / (2 * heads);
    const dim3 grid((unsigned)plan->append_groups.size(), (unsigned)blocks);
    auto kernel = steps ? kv8_step_kernel<T, D, STYLE> : kv8_append_kernel<T, D, STYLE, 1, false>;
    if constexpr (STYLE < 0) {
        if (!steps && streams) kernel = kv8_append_kernel<T, D, STYLE, 1, true>;
    } else {
        if (!steps && two) kernel = kv8_append_kernel<T, D, STYLE, 2, false>;
        if (!steps && streams) kernel = kv8_append_kernel<T, D, STYLE, 2, true>;
    }
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
    // two heads a wavefront where there are enough pages to fill the GPU all the same: 69 K tokens, 8 heads
    // 86.8 us (one head 94.0), 8 K 9.1 (9.3), 2.4 K 4.6 (4.4), 600 3.3 (2.9)
    const bool two = (int64_t)plan->append_groups.size() * plan->pool.num_kv_heads >= 4000;
    const int hb = two ? 2 : 1;
    auto pick = [&](auto heads) {
        constexpr int HB = decltype(heads)::value;
        return plan->pool.head_dim == 128
                   ? (f ? kv8_read_kernel<F16, 128, HB> : kv8_read_kernel<BF16, 128, HB>)
                   : (f ? kv8_read_kernel<F16, 64, HB> : kv8_read_kernel<BF16, 64, HB>);
    };
    auto kernel = two ? pick(std::integral_constant<int, 2>{}) : pick(std::integral_constant<int, 1>{});
    const dim3 grid((unsigned)plan->append_groups.size(),
                    (unsigned)((plan->pool.num_kv_heads + hb - 1) / hb));
    hipLaunchKernelGGL(kernel, grid, dim3(128), 0, stream, dl.append_groups, p, page_table,
                       plan->max_pages_per_req, plan->pool.num_kv_heads, (uint16_t *)k_rows,
                       (uint16_t *)v_rows);
    return hipGetLastError();
}

}  // namespace pv
