// Rows of queries or keys, normalised and rotated, in the layout that reads and writes them best: what
// the appends into 16-bit and into 8-bit pools share (gfx950 only).
#pragma once

#include "pv_device.h"

namespace pv {

// A lane holds chunks c and c + D/16 (of 8 dimensions) of a
// row, partners of a rotation, so that the D/16 lanes of a row read and write 16 bytes side by side.
template <int D, int STYLE>
struct ChunkAngles {
    f32x4 c[2], s[2];
    __device__ __forceinline__ void load(const float *cs, int lane_c)
    {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float *at = cs + (STYLE == 1 ? 8 * lane_c + 4 * k : 4 * lane_c + k * (D / 4));
            c[k] = *reinterpret_cast<const f32x4 *>(at);
            s[k] = *reinterpret_cast<const f32x4 *>(at + D / 2);
        }
    }
};

template <typename T, int D, int STYLE>
__device__ __forceinline__ void norm_rotate_chunks(u32x4 (&raw)[2], bool norm,
                                                   const u32x4 (&weight)[2], float eps,
                                                   const ChunkAngles<D, STYLE> &angle)
{
    float x[2][8], y[2][8];
    unpack8<T>(raw[0], x[0]);
    unpack8<T>(raw[1], x[1]);
    if (norm) {
        const float r = norm_factor<D>(sum_squares(x[0]) + sum_squares(x[1]), eps);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float w[8];
            unpack8<T>(weight[i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] * r * w[e];
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (STYLE == 1)  // dimensions i and i + D/2
                rotate_pair(x[0][4 * k + e], x[1][4 * k + e], angle.c[k][e], angle.s[k][e],
                            y[0][4 * k + e], y[1][4 * k + e]);
            else  // dimensions 2i and 2i + 1
                rotate_pair(x[k][2 * e], x[k][2 * e + 1], angle.c[k][e], angle.s[k][e], y[k][2 * e],
                            y[k][2 * e + 1]);
        }
    raw[0] = pack8<T>(y[0]);
    raw[1] = pack8<T>(y[1]);
}

// HEADS heads of TOKENS tokens a lane (of one wavefront): token t of the lane is j0 + t * 64 / (D/16) of the
// group if that exists, `row` the element of its head 0 there, heads `step` elements apart.
template <typename T, int D, int STYLE, int HEADS, int TOKENS, bool STREAM>
__device__ __forceinline__ void rotate_q(const AppendGroup &g, int j0, int64_t token_step,
                                         int64_t row, int64_t step, int heads, const uint16_t *q_in,
                                         uint16_t *q_out, const uint16_t *weight, float eps,
                                         const float *cos_sin)
{
    constexpr int LPR = D / 16;
    const int c = lane_id() % LPR;
    u32x4 rows[TOKENS][HEADS][2], w[2];
    ChunkAngles<D, STYLE> angle[TOKENS];
    int64_t at[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        const int j = min(j0 + t * (64 / LPR), g.count - 1);
        at[t] = row + j * token_step + 8 * c;
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const uint16_t *from = q_in + at[t] + (i < heads ? i : 0) * step;
            rows[t][i][0] = load16_as<STREAM>(from);
            rows[t][i][1] = load16_as<STREAM>(from + D / 2);
        }
        angle[t].load(cos_sin + (int64_t)(g.t_begin + j) * D, c);
    }
    if (weight) {
        w[0] = load16(weight + 8 * c);
        w[1] = load16(weight + D / 2 + 8 * c);
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t)
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            norm_rotate_chunks<T, D, STYLE>(rows[t][i], weight != nullptr, w, eps, angle[t]);
            if (i < heads && j0 + t * (64 / LPR) < g.count) {
                uint16_t *to = q_out + at[t] + i * step;
                *reinterpret_cast<u32x4 *>(to) = rows[t][i][0];
                *reinterpret_cast<u32x4 *>(to + D / 2) = rows[t][i][1];
            }
        }
}

// Of a batch's steps of one token: the first of the lane's two heads out of 128 / (D/16) that a wavefront
// takes from h0 on, clamped to the last one there is, and how many of the two exist.
template <int D>
struct StepHeads {
    static constexpr int kEach = 64 / (D / 16), kHeads = 2 * kEach;
    int first, count;
    __device__ __forceinline__ StepHeads(int h0, int num_heads)
    {
        const int h = h0 + lane_id() / (D / 16);
        first = min(h, num_heads - 1);
        count = h < num_heads ? (num_heads - h + kEach - 1) / kEach : 0;
    }
};

}  // namespace pv
