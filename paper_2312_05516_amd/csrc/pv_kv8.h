// Codes and scales of the 8-bit pools (gfx950 only).
//
// A code is an e4m3 value: sign, 4 exponent bits (bias 7), 3 of mantissa, no infinity, NaN =
// 0x7F / 0xFF, largest 448, smallest 2^-9.  A block, one (page, KV head) of K or of V, has a scale
// 2^e, held as the byte e + 127.  e is limited so that every code * 2^e is a value of the pool's
// 16-bit type: f16 -15 .. 8 (2^-9 * 2^-15 is its smallest subnormal), bf16 -117 .. 120 (2^-9 *
// 2^-117 is its smallest normal value); with the largest e codes end at 240, because 256 * 2^e
// would be past the type's range.  So reading a code back is exact, and attention over the codes
// is attention over the 16-bit values that pv_kv8_read_planned returns.
//
// Scales are powers of two because a floating-point code loses nothing by that (its relative
// precision does not depend on the scale), x * 2^-e is exact, so that codes do not depend on the
// order or precision of any arithmetic, and a block whose scale grows keeps its codes' values
// exactly but for those that become subnormal.
#pragma once

#include "pv_device.h"

namespace pv {

// Pool pointers of the 8-bit calls, device side.
struct Kv8Ptrs {
    uint8_t *k, *v, *k_scales, *v_scales;
};

// Byte offsets inside a (page, head) tile of 16 * D codes.  K: the 16 dimensions of a chunk of one
// slot are one lane's 16 bytes (two matrix-core operands); 4 slots x 64 dimensions are 256
// contiguous bytes, what 16 lanes of the 16-row kernel read at once.  V: the 16 slots of one
// dimension are 16 bytes.
template <int D>
__device__ __forceinline__ int kv8_k_chunk(int slot, int chunk)
{
    return (slot >> 2) * (4 * D) + chunk * 64 + (slot & 3) * 16;
}

__device__ __forceinline__ float exp2_scale(int byte)  // 2^(byte - 127) for bytes 1 .. 254
{
    return __builtin_bit_cast(float, (uint32_t)byte << 23);
}

template <typename T>
struct Kv8;

template <>
struct Kv8<F16> {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static constexpr int kMinExp = -15, kMaxExp = 8;
    static constexpr uint32_t kTop = 0x7B80u;  // 240 * 2^8
    // codes 2h, 2h+1 of a word times the scale, as a packed pair (exact)
    template <bool HI>
    static __device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale)
    {
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HI));
    }
    // the codes of a packed pair divided by the scale (nearest even) into that half of `old`
    template <bool HI>
    static __device__ __forceinline__ uint32_t encode2(uint32_t old, uint32_t xy, float scale)
    {
        typedef short s2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(
                          __builtin_bit_cast(s2, old), __builtin_bit_cast(pair, xy), scale, HI));
    }
};

template <>
struct Kv8<BF16> {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static constexpr int kMinExp = -117, kMaxExp = 120;
    static constexpr uint32_t kTop = 0x7F70u;  // 240 * 2^120
    template <bool HI>
    static __device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale)
    {
        return __builtin_bit_cast(uint32_t,
                                  __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
    }
    template <bool HI>
    static __device__ __forceinline__ uint32_t encode2(uint32_t old, uint32_t xy, float scale)
    {
        typedef short s2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(
            uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
                          __builtin_bit_cast(s2, old), __builtin_bit_cast(pair, xy), scale, HI));
    }
};

// 8 codes (two words) -> the 8 values of a matrix-core operand
template <typename T>
__device__ __forceinline__ u32x4 decode8(uint32_t lo, uint32_t hi, float scale)
{
    return u32x4{Kv8<T>::template decode2<false>(lo, scale), Kv8<T>::template decode2<true>(lo, scale),
                 Kv8<T>::template decode2<false>(hi, scale), Kv8<T>::template decode2<true>(hi, scale)};
}

// 0xFF in the first n bytes of a word (n may be below 0 or above 4)
__device__ __forceinline__ uint32_t codes_in_front(int n)
{
    return (uint32_t)((1ull << (8 * min(max(n, 0), 4))) - 1);
}

// 0x80 in the bytes of a word that are NaN
__device__ __forceinline__ uint32_t nan_codes(uint32_t codes)
{
    return ((codes & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Magnitudes of a packed pair of 16-bit values as integers, which order as the values do; an
// infinity or NaN counts as zero.
template <typename T>
__device__ __forceinline__ uint32_t finite_magnitudes(uint32_t xy)
{
    uint32_t lo = xy & 0x7FFFu, hi = xy & 0x7FFF0000u;
    lo = lo >= T::kExponent ? 0u : lo;
    hi = hi >= (T::kExponent << 16) ? 0u : hi;
    return lo | hi;
}
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t a, uint32_t b)
{
    typedef unsigned short u2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u2, a),
                                                                  __builtin_bit_cast(u2, b)));
}

// The largest magnitudes (of either half) among LANES neighbouring lanes, in all of them
template <int LANES>
__device__ __forceinline__ uint32_t max_of_lanes(uint32_t mag)
{
    mag = max_magnitudes(mag, other_lane<1>(mag));
    if constexpr (LANES > 2) mag = max_magnitudes(mag, other_lane<2>(mag));
    if constexpr (LANES > 4) mag = max_magnitudes(mag, other_lane<4>(mag));
    if constexpr (LANES > 8) mag = max_magnitudes(mag, other_lane<8>(mag));
    if constexpr (LANES > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(mag, mag, false, false);
        mag = max_magnitudes(r[0], r[1]);
    }
    if constexpr (LANES > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(mag, mag, false, false);
        mag = max_magnitudes(r[0], r[1]);
    }
    return mag;
}

// The least e in the type's range with a <= 448 * 2^e, `magnitude` being the bits of a.
template <typename T>
__device__ __forceinline__ int needed_exponent(uint32_t magnitude)
{
    float a, unused;
    T::unpack2(magnitude, a, unused);
    const uint32_t bits = __builtin_bit_cast(uint32_t, a);
    // a = 1.m * 2^x  <=  1.75 * 2^(8 + e)
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return max(e, Kv8<T>::kMinExp);  // no finite value needs more than kMaxExp
}

// with the largest scale: finite values of a packed pair no larger than kTop
template <typename T>
__device__ __forceinline__ uint32_t limit_to_top(uint32_t xy)
{
    const uint32_t lo = xy & 0x7FFFu, hi = (xy >> 16) & 0x7FFFu;
    if (lo > Kv8<T>::kTop && lo < T::kExponent) xy = (xy & 0xFFFF8000u) | Kv8<T>::kTop;
    if (hi > Kv8<T>::kTop && hi < T::kExponent) xy = (xy & 0x8000FFFFu) | (Kv8<T>::kTop << 16);
    return xy;
}

// Four codes of a scale 2^from rounded anew for the scale 2^to, to > from.  (Their values, without
// scales, are exact in f16.)
__device__ __forceinline__ uint32_t rescale4(uint32_t codes, int from, int to)
{
    const float by = exp2_scale(127 + min(to - from, 100));  // beyond that everything is zero
    uint32_t r = Kv8<F16>::encode2<false>(0u, Kv8<F16>::decode2<false>(codes, 1.f), by);
    return Kv8<F16>::encode2<true>(r, Kv8<F16>::decode2<true>(codes, 1.f), by);
}

}  // namespace pv
