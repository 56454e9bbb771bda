// kv4.cuh -- the 4-bit KV cache: its format and the quantiser, for the kernels that write and read it.
//
// A head's D values of a slot are quantised in groups of 32.  A group x has
//   lo = min(x, 0), hi = max(x, 0)
//   s  = the smallest number of 4 significant bits that is >= (hi - lo) / 15, at least 2^-126
//   z  = rint(-lo / s)                            0 .. 15
//   c  = min(max(rint(x / s) + z, 0), 15)         the code
// and stands for (c - z) s.  |c - z| <= 15 and s have 4 significant bits each, so the product is a
// bf16 exactly (up to overflow, from |x| of about 2^127): there is no rounding in reading a cache, and a
// kernel may take c s and z s apart.  A group that holds an infinity or a NaN has c = z = 0 and s = NaN, and
// reads as NaN.
//
// codes  [B][Hkv][Lp][D/2] bytes (Lp: max_len rounded up to kKv4Slots): words of 8 values, the code of
//        value j at bit (0, 16, 4, 20, 8, 24, 12, 28)[j], so that a shift and one masked OR make a
//        pair of neighbours (the order of the W4BF16 tiles)
// scales [B][Hkv][Lp][D/32] 16 bits: s as a bf16, whose four lowest bits are zero, with z in their place
#pragma once

#include <cuda_bf16.h>

#include <cstdint>

namespace attn {

constexpr int kKv4Group = 32;
constexpr uint32_t kKv4ScaleMask = 0x7FF0u, kKv4NanScale = 0x7FF0u;

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The larger of each pair, NaN where either is.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight values of a word as four bf16 pairs (values 2i and 2i + 1 in the halves of out[i]): 128 + c less 128 + z,
// times s, all of it exact.
__device__ __forceinline__ void kv4_values(uint32_t w, uint32_t m, uint32_t (&out)[4]) {
    const uint32_t m2 = m * 0x10001u, s = m2 & 0x7FF07FF0u, z = (m2 & 0x000F000Fu) | 0x43004300u;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = mul2(sub2(((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u, z), s);
}

// The scale (bits of a bf16, low four bits zero) of a group with extremes -neg <= 0 <= hi: the next number of 4
// bits from a quotient that is 1 or 2 parts in 2^22 too small is s or the one before it, and the one before where
// it leaves 7.5 s < (hi + neg) / 2, told from the larger half less 7.5 s, which is exact where that decides.
// (Halves, so that the sum does not overflow; what a subnormal loses by it is under the least scale.)
__device__ __forceinline__ uint32_t kv4_scale_of(float hi, float neg) {
    const float h = hi * 0.5f, l = neg * 0.5f;
    uint32_t up = (__float_as_uint(__fmul_rn(__fadd_rn(h, l), 0.133333295f)) + 0xFFFFFu) & 0xFFF00000u;
    if (__fsub_rn(fmaxf(h, l), __fmul_rn(__uint_as_float(up), 7.5f)) > -fminf(h, l)) up += 0x00100000u;
    return max(up, 0x00800000u) >> 16;
}

// rint(x / s) + 0x4B400000 for a bf16 x and the reciprocal inv of a scale, good to a few parts in 2^23: x / s (8 bits
// over 4) is a tie or at least 2^-10 away from one, so x * inv rounded to a multiple of 2^-11 (by adding 1.5 * 2^12) is
// the tie itself or on its quotient's side of it, and adding on to 1.5 * 2^23 leaves the integer in the low bits.
__device__ __forceinline__ int kv4_round(float x, float inv) {
    return __float_as_int(__fadd_rn(__fmaf_rn(x, inv, 6144.0f), 12582912.0f - 6144.0f));
}
constexpr int kKv4Round = 0x4B400000;

// (hi, -lo) of eight values, given as bf16 pairs, in the halves of the result: at least 0, NaN where a value is.
__device__ __forceinline__ uint32_t kv4_extremes(const uint32_t (&w)[4]) {
    constexpr uint32_t kSign = 0x80008000u;
    const uint32_t hi = max2(max2(w[0], w[1]), max2(w[2], w[3]));
    const uint32_t lo = max2(max2(w[0] ^ kSign, w[1] ^ kSign), max2(w[2] ^ kSign, w[3] ^ kSign));
    return max2(max2(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632)), 0u);
}

// The scale and zero point of a group with those extremes, and the reciprocal of the scale.
__device__ __forceinline__ uint32_t kv4_group(uint32_t extremes, float& inv) {
    const uint32_t s = kv4_scale_of(bf_lo(extremes), bf_hi(extremes));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__uint_as_float(s << 16)));  // 2^-126 <= s < 2^126
    const bool odd = (extremes & 0x7F80u) == 0x7F80u || (extremes & 0x7F800000u) == 0x7F800000u;
    return odd ? kKv4NanScale : s | static_cast<uint32_t>(kv4_round(bf_hi(extremes), inv) - kKv4Round);
}

// The code of x in a group: rint(x / s) + z, which is not negative (x >= lo), and at most 15 (both
// roundings up may make 16).
__device__ __forceinline__ uint32_t kv4_code(float x, float inv, int z) {
    return static_cast<uint32_t>(min(kv4_round(x, inv) + (z - kKv4Round), 15));
}

// Eight neighbours, as bf16 pairs, of a group that four consecutive lanes of a full warp hold: the word of their
// codes, and the group's scale and zero point.
__device__ __forceinline__ uint32_t kv4_quantise8(const uint32_t (&x)[4], uint32_t& scale) {
    uint32_t e = kv4_extremes(x);
    e = max2(e, __shfl_xor_sync(0xFFFFFFFFu, e, 1));
    e = max2(e, __shfl_xor_sync(0xFFFFFFFFu, e, 2));
    float inv;
    scale = kv4_group(e, inv);
    if (scale == kKv4NanScale) return 0;
    const int z = static_cast<int>(scale & 15u);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w |= (kv4_code(bf_lo(x[i]), inv, z) | kv4_code(bf_hi(x[i]), inv, z) << 16) << (4 * i);
    return w;
}
#endif

}  // namespace attn
