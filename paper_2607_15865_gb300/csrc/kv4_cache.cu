// kv4_cache.cu -- writing and reading the 4-bit KV cache (format: kv4.cuh).
//
//   append  new k (rotated, as K1 rotates it, and rounded to bf16) and v, quantised into their slots
//   read    slots back to bf16
//   fill    both at once, for the prefill stages: the chunk is appended and, with the history before
//           it, written as bf16 to a workspace that flash_fwd then reads
//
// All of it is bandwidth: 4 D bytes of new k and v in and 9/8 D out per token and kv head for
// append, the reverse for read.
#include "internal.h"
#include "kv4.cuh"
#include "sm100_ptx.cuh"

namespace attn {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf_lo(w[i]);
        x[2 * i + 1] = bf_hi(w[i]);
    }
}

// The word of a row of D values at value index j (a multiple of 8), and its group's scale; with `out` (a
// row of bf16) also the values that they stand for.
__device__ __forceinline__ void put(const float (&x)[8], int j, bool mine, uint8_t* codes, uint16_t* scales,
                                    uint16_t* out) {
    uint32_t scale;
    const uint32_t w = kv4_quantise8(x, scale);
    if (!mine) return;
    *reinterpret_cast<uint32_t*>(codes + j / 2) = w;
    if (j % kKv4Group == 0) scales[j / kKv4Group] = static_cast<uint16_t>(scale);
    if (out != nullptr) {
        uint32_t v[4];
        kv4_values(w, scale, v);
        *reinterpret_cast<uint4*>(out + j) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// One thread per 16 values of k and of v (8 and their RoPE partners D / 2 further) of a (token, kv head).
template <int D>
__device__ __forceinline__ void append_unit(long long u, const Kv4New& a, int Hkv, int max_len, int lp, const float* cos_tab,
                                            const float* sin_tab, const Kv4Cache& c, const Kv4Plain& plain, int* err) {
    constexpr int PARTS = D / 16;
    const long long n = static_cast<long long>(a.batch) * a.chunk * Hkv * PARTS;
    const bool in = u < n;
    if (!in) u = n - 1;  // whole warps take part in the group reductions
    const int part = static_cast<int>(u % PARTS);
    const long long row = u / PARTS;  // (sequence, token, head)
    const int g = static_cast<int>(row % Hkv);
    const int i = static_cast<int>(row / Hkv % a.chunk);
    const int b = static_cast<int>(row / Hkv / a.chunk);
    int hist = a.hist;
    bool mine = in;
    if (a.d_hist != nullptr) {
        hist = a.d_hist[b];
        if (hist < 0 || hist > max_len - a.chunk) {
            if (in && part == 0 && g == 0 && i == 0) atomicOr(err, kDevErrHistRange);
            mine = false;
            hist = 0;
        }
    }
    const int p = hist + i, j = 8 * part;
    const size_t src = static_cast<size_t>(row) * D + j;
    const size_t slot = (static_cast<size_t>(b) * Hkv + g) * lp + p;
    const size_t prow = (static_cast<size_t>(b) * Hkv + g) * plain.rows + p;
    float xa[8], xb[8], cs[8], sn[8], ya[8], yb[8];
    unpack8(*reinterpret_cast<const uint4*>(a.k + src), xa);
    unpack8(*reinterpret_cast<const uint4*>(a.k + src + D / 2), xb);
    const uint4 va = *reinterpret_cast<const uint4*>(a.v + src), vb = *reinterpret_cast<const uint4*>(a.v + src + D / 2);
    const float4* ct = reinterpret_cast<const float4*>(cos_tab + static_cast<size_t>(p) * (D / 2) + j);
    const float4* st = reinterpret_cast<const float4*>(sin_tab + static_cast<size_t>(p) * (D / 2) + j);
    *reinterpret_cast<float4*>(cs) = ct[0];
    *reinterpret_cast<float4*>(cs + 4) = ct[1];
    *reinterpret_cast<float4*>(sn) = st[0];
    *reinterpret_cast<float4*>(sn + 4) = st[1];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        ya[e] = round_bf16(__fsub_rn(__fmul_rn(xa[e], cs[e]), __fmul_rn(xb[e], sn[e])));
        yb[e] = round_bf16(__fadd_rn(__fmul_rn(xb[e], cs[e]), __fmul_rn(xa[e], sn[e])));
    }
    uint8_t* kc = c.k_codes + slot * (D / 2);
    uint8_t* vc = c.v_codes + slot * (D / 2);
    uint16_t* ks = c.k_scales + slot * (D / kKv4Group);
    uint16_t* vs = c.v_scales + slot * (D / kKv4Group);
    uint16_t* ko = plain.k == nullptr ? nullptr : plain.k + prow * D;
    uint16_t* vo = plain.v == nullptr ? nullptr : plain.v + prow * D;
    put(ya, j, mine, kc, ks, ko);
    put(yb, j + D / 2, mine, kc, ks, ko);
    unpack8(va, xa);
    unpack8(vb, xb);
    put(xa, j, mine, vc, vs, vo);
    put(xb, j + D / 2, mine, vc, vs, vo);
}

// One thread per word of 8 values, of k and of v, of slots first .. first + count - 1.
template <int D>
__device__ __forceinline__ void read_unit(long long u, int first, int count, int heads, int lp, const Kv4Cache& c,
                                          const Kv4Plain& plain) {
    constexpr int WORDS = D / 8;
    if (u >= static_cast<long long>(heads) * count * WORDS) return;
    const int word = static_cast<int>(u % WORDS);
    const long long r = u / WORDS;
    const int i = static_cast<int>(r % count), h = static_cast<int>(r / count);
    const size_t slot = static_cast<size_t>(h) * lp + first + i;
    const size_t out = (static_cast<size_t>(h) * plain.rows + i) * D + 8 * word;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const uint8_t* codes = t ? c.v_codes : c.k_codes;
        const uint16_t* scales = t ? c.v_scales : c.k_scales;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + slot * (D / 2) + 4 * word);
        uint32_t v[4];
        kv4_values(w, scales[slot * (D / kKv4Group) + word / 4], v);
        *reinterpret_cast<uint4*>((t ? plain.v : plain.k) + out) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(Kv4New a, int Hkv, int max_len, int lp,
                                                              const float* __restrict__ cos_tab,
                                                              const float* __restrict__ sin_tab, Kv4Cache c, Kv4Plain plain,
                                                              int append_blocks, int* __restrict__ err) {
    // A dependent launch: it reads and writes only after the stream's previous kernel, and the kernel after it
    // (flash_fwd, whose prologue reads q) may be resident by then.
    griddep_wait();
    griddep_launch_dependents();
    const int block = static_cast<int>(blockIdx.x);
    if (block < append_blocks)
        append_unit<D>(static_cast<long long>(block) * kThreads + threadIdx.x, a, Hkv, max_len, lp, cos_tab, sin_tab, c,
                       plain, err);
    else  // the history in front of the chunk, to the workspace
        read_unit<D>(static_cast<long long>(block - append_blocks) * kThreads + threadIdx.x, 0, a.hist, a.batch * Hkv, lp,
                     c, plain);
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(int first, int count, int heads, int lp, Kv4Cache c,
                                                            Kv4Plain plain) {
    griddep_wait();
    griddep_launch_dependents();
    read_unit<D>(static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, first, count, heads, lp, c, plain);
}

cudaLaunchConfig_t dependent(long long blocks, cudaStream_t st, cudaLaunchAttribute* attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

long long blocks_for(long long units) { return (units + kThreads - 1) / kThreads; }

}  // namespace

cudaError_t launch_kv4_append(const Shape& s, const Kv4New& a, const float* cos_tab, const float* sin_tab, const Kv4Cache& c,
                              const Kv4Plain& plain, int* err, cudaStream_t st) {
    const long long tokens = static_cast<long long>(a.batch) * a.chunk;
    const long long append = blocks_for(tokens * s.n_kv_heads * (s.head_dim / 16));
    const long long read =
        plain.k == nullptr ? 0 : blocks_for(static_cast<long long>(a.batch) * s.n_kv_heads * a.hist * (s.head_dim / 8));
    if (append + read > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(append + read, st, &attr);
    return cudaLaunchKernelEx(&cfg, s.head_dim == 128 ? kv4_append_kernel<128> : kv4_append_kernel<64>, a, s.n_kv_heads,
                              s.max_len, kv4_slots(s.max_len), cos_tab, sin_tab, c, plain, static_cast<int>(append), err);
}

cudaError_t launch_kv4_read(const Shape& s, int first, int count, const Kv4Cache& c, const Kv4Plain& plain,
                            cudaStream_t st) {
    const int heads = s.batch * s.n_kv_heads;
    const long long blocks = blocks_for(static_cast<long long>(heads) * count * (s.head_dim / 8));
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(blocks, st, &attr);
    return cudaLaunchKernelEx(&cfg, s.head_dim == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>, first, count, heads,
                              kv4_slots(s.max_len), c, plain);
}

}  // namespace attn
