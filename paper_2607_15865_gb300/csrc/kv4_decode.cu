// kv4_decode.cu -- decode attention over a 4-bit KV cache (format: kv4.cuh), the simple form: a CTA per
// (new token, query head) walks the token's slots, a warp per slot, in f32.
#include <cmath>

#include "internal.h"
#include "kv4.cuh"

namespace attn {
namespace {

constexpr int kWarps = 4;

__device__ __forceinline__ float bf16_at(const uint16_t* p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }

template <int D>
__global__ void __launch_bounds__(32 * kWarps) kv4_decode_kernel(const uint16_t* __restrict__ q, Kv4Cache c,
                                                                 const int32_t* __restrict__ d_hist, int ntok, int Hq,
                                                                 int Hkv, int max_len, int lp, float scale_log2,
                                                                 const float* __restrict__ cos_tab,
                                                                 const float* __restrict__ sin_tab,
                                                                 uint16_t* __restrict__ out) {
    constexpr int E = D / 32;  // values per lane
    const int h = blockIdx.x % Hq, i = blockIdx.x / Hq, b = blockIdx.y;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int hist = d_hist[b];
    if (hist < 0 || hist > max_len - ntok) return;
    const int p = hist + i;
    const size_t row = ((static_cast<size_t>(b) * ntok + i) * Hq + h) * D;
    float qr[E], acc[E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int d = lane * E + e, j = d % (D / 2);
        const float cs = cos_tab[static_cast<size_t>(p) * (D / 2) + j], sn = sin_tab[static_cast<size_t>(p) * (D / 2) + j];
        const float x = bf16_at(q + row + d), y = bf16_at(q + row + (d + D / 2) % D);
        const float r = d < D / 2 ? __fsub_rn(__fmul_rn(x, cs), __fmul_rn(y, sn)) : __fadd_rn(__fmul_rn(x, cs), __fmul_rn(y, sn));
        qr[e] = __bfloat162float(__float2bfloat16_rn(r));
    }
    const size_t slot0 = (static_cast<size_t>(b) * Hkv + h / (Hq / Hkv)) * lp;
    const int grp = lane * E / kKv4Group, word = lane * E / 8;
    auto value = [&](const uint8_t* codes, const uint16_t* scales, size_t slot, int e) {
        const int j = (lane * E + e) % 8;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + slot * (D / 2) + 4 * word);
        const uint32_t s = scales[slot * (D / kKv4Group) + grp];
        const float code = static_cast<float>((w >> (4 * (j >> 1) + 16 * (j & 1))) & 15u);
        return (code - static_cast<float>(s & 15u)) * kv4_scale(s);
    };
    for (int k = warp; k <= p; k += kWarps) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += qr[e] * value(c.k_codes, c.k_scales, slot0 + k, e);
#pragma unroll
        for (int mask = 16; mask > 0; mask >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, mask);
        s *= scale_log2;
        const float mn = fmaxf(m, s), al = exp2f(m - mn), w = exp2f(s - mn);
        l = l * al + w;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * al + w * value(c.v_codes, c.v_scales, slot0 + k, e);
        m = mn;
    }
    __shared__ float sm[kWarps], sl[kWarps], so[kWarps][D];
    if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) so[warp][lane * E + e] = acc[e];
    __syncthreads();
    if (threadIdx.x >= D) return;
    float mx = sm[0], o = 0.f, lt = 0.f;  // warp 0 has slot 0
    for (int w = 1; w < kWarps; ++w) mx = fmaxf(mx, sm[w]);
    for (int w = 0; w < kWarps; ++w) {
        if (sl[w] == 0.f) continue;
        const float f = exp2f(sm[w] - mx);
        o += f * so[w][threadIdx.x];
        lt += f * sl[w];
    }
    out[row + threadIdx.x] = __bfloat16_as_ushort(__float2bfloat16_rn(o / lt));
}

}  // namespace

cudaError_t launch_kv4_decode(const Shape& s, const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                              const int32_t* d_hist, int ntok, const Kv4Cache& c, const float* cos_tab,
                              const float* sin_tab, uint16_t* out, int* err, cudaStream_t st) {
    const Kv4New a{k_new, v_new, d_hist, 0, ntok, s.batch};
    const cudaError_t e = launch_kv4_append(s, a, cos_tab, sin_tab, c, Kv4Plain{nullptr, nullptr, 0}, err, st);
    if (e != cudaSuccess) return e;
    const float scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim)));
    const dim3 grid(static_cast<unsigned>(ntok * s.n_q_heads), static_cast<unsigned>(s.batch));
    const auto fn = s.head_dim == 128 ? kv4_decode_kernel<128> : kv4_decode_kernel<64>;
    fn<<<grid, 32 * kWarps, 0, st>>>(q, c, d_hist, ntok, s.n_q_heads, s.n_kv_heads, s.max_len, kv4_slots(s.max_len),
                                     scale_log2, cos_tab, sin_tab, out);
    return cudaGetLastError();
}

}  // namespace attn
