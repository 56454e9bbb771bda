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
__device__ __forceinline__ float kv4_scale(uint32_t m) { return __uint_as_float((m & kKv4ScaleMask) << 16); }

// Eight values of a word as four bf16 pairs (values 2i and 2i + 1 in the halves of out[i]).
__device__ __forceinline__ void kv4_values(uint32_t w, uint32_t m, uint32_t (&out)[4]) {
    const float s = kv4_scale(m), z = static_cast<float>(m & 15u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = static_cast<float>((w >> (4 * i)) & 15u), hi = static_cast<float>((w >> (16 + 4 * i)) & 15u);
        const __nv_bfloat162 p = __floats2bfloat162_rn((lo - z) * s, (hi - z) * s);
        out[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
}

// The scale (bits of a bf16, low four bits zero) of a group with extremes lo <= 0 <= hi.  The halves
// are exact (what a subnormal loses is under the least scale), and (hi - lo) / 15 rounds to a number of 4 bits
// where it is one or where the difference loses a far smaller lo or hi; hi / 2 - 7.5 s, which is exact
// near that, tells those apart.
__device__ __forceinline__ uint32_t kv4_scale_of(float lo, float hi) {
    const float h = hi * 0.5f, l = lo * 0.5f;
    uint32_t up = (__float_as_uint(__fdiv_rn(__fsub_rn(h, l), 7.5f)) + 0xFFFFFu) & 0xFFF00000u;
    if (__fsub_rn(h, __fmul_rn(__uint_as_float(up), 7.5f)) > l) up += 0x00100000u;
    return max(up, 0x00800000u) >> 16;
}

// rint(x / s) for a bf16 x and the reciprocal inv of a scale: x / s (8 bits over 4) is a tie or at least
// 2^-10 away from one, so x * inv rounded to a multiple of 2^-11 (by adding and taking off
// 1.5 * 2^12) is the tie itself or on its quotient's side of it.
__device__ __forceinline__ int kv4_round(float x, float inv) {
    const float t = __fsub_rn(__fadd_rn(__fmul_rn(x, inv), 6144.0f), 6144.0f);
    return __float_as_int(__fadd_rn(t, 12582912.0f)) - 0x4B400000;  // 1.5 * 2^23: the integer in the low bits
}

// Eight neighbours of a group that four consecutive lanes of a full warp hold (lane & 3 = the word
// of the group): the word of their codes, and the group's scale and zero point.
__device__ __forceinline__ uint32_t kv4_quantise8(const float (&x)[8], uint32_t& scale) {
    float lo = 0.f, hi = 0.f;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
        odd |= (__float_as_uint(x[j]) & 0x7F800000u) == 0x7F800000u;
    }
#pragma unroll
    for (int mask = 1; mask <= 2; mask <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, mask));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, mask));
    }
    const uint32_t odds = __ballot_sync(0xFFFFFFFFu, odd);
    if ((odds >> (threadIdx.x & 28)) & 15u) {
        scale = kKv4NanScale;
        return 0;
    }
    const uint32_t s = kv4_scale_of(lo, hi);
    const float inv = __frcp_rn(__uint_as_float(s << 16));
    const int z = kv4_round(-lo, inv);
    scale = s | static_cast<uint32_t>(z);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = min(max(kv4_round(x[j], inv) + z, 0), 15);
        w |= static_cast<uint32_t>(c) << (4 * (j >> 1) + 16 * (j & 1));
    }
    return w;
}
#endif

}  // namespace attn
