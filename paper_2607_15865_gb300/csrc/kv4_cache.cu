// kv4_cache.cu -- writing and reading the 4-bit KV cache (format: kv4.cuh).
//
//   append  new k (rotated, as K1 rotates it, and rounded to bf16) and v, quantised into their slots
//   read    slots back to bf16
//   fill    both at once, for the prefill stages: the chunk is appended and, with the history before
//           it, written as bf16 to a workspace that flash_fwd then reads
//
// Bytes per token and kv head: 4 D of new k and v in and 9/8 D out for append (and a table row per token), the
// reverse for read.  Measured in a graph, 8 heads of 128 values, rotating caches:
//   append  512 tokens 2.1 us, 4096 5.9 us, 16384 21.3 us (86 MB and 8 MB of tables, 4.4 TB/s): between issue (63% of
//           the cycles, cold; the extremes of the groups, the scales and the codes) and the wait for a thread's one round
//           of loads (28% of a warp's time); 5 CTAs of 48 registers per SM; at 40 registers, 6 CTAs, 4096 tokens took
//           6.6 us, at 32 9.3 us, both with spills
//   read    2048 slots 2.4 us, 32767 27.7 us (172 MB, 6.2 TB/s, 92% of the copy bandwidth): memory.  A thread has eight
//           words and their scales in flight
#include <algorithm>

#include "internal.h"
#include "kv4.cuh"
#include "sm100_ptx.cuh"

namespace attn {
namespace {

constexpr int kThreads = 256;

// The word of a row of D values at value index j (a multiple of 8), and its group's scale; with `out` (a
// row of bf16) also the values that they stand for.
__device__ __forceinline__ void put(const uint4& x, int j, bool mine, uint8_t* codes, uint16_t* scales, uint16_t* out) {
    const uint32_t pairs[4] = {x.x, x.y, x.z, x.w};
    uint32_t scale;
    const uint32_t w = kv4_quantise8(pairs, scale);
    if (!mine) return;
    *reinterpret_cast<uint32_t*>(codes + j / 2) = w;
    if (j % kKv4Group == 0) scales[j / kKv4Group] = static_cast<uint16_t>(scale);
    if (out != nullptr) {
        uint32_t v[4];
        kv4_values(w, scale, v);
        *reinterpret_cast<uint4*>(out + j) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// RoPE of two pairs: values j, j + 1 in x and their partners in y.
__device__ __forceinline__ void turn(uint32_t& x, uint32_t& y, float c0, float c1, float s0, float s1) {
    const float x0 = bf_lo(x), x1 = bf_hi(x), y0 = bf_lo(y), y1 = bf_hi(y);
    x = pack2(__fsub_rn(__fmul_rn(x0, c0), __fmul_rn(y0, s0)), __fsub_rn(__fmul_rn(x1, c1), __fmul_rn(y1, s1)));
    y = pack2(__fadd_rn(__fmul_rn(y0, c0), __fmul_rn(x0, s0)), __fadd_rn(__fmul_rn(y1, c1), __fmul_rn(x1, s1)));
}

// One thread per 16 values of k and of v (8 and their RoPE partners D / 2 further) of a (token, kv head).
struct AppendCut {
    FastDiv heads, chunk;
    int units, lp, blocks;
};
template <int D>
__device__ __forceinline__ void append_unit(int u, const Kv4New& a, const AppendCut& cut, const float* cos_tab,
                                            const float* sin_tab, const Kv4Cache& c, const Kv4Plain& plain) {
    constexpr int PARTS = D / 16;
    const bool mine = u < cut.units;
    if (!mine) u = cut.units - 1;  // whole warps take part in the group reductions
    const int part = u % PARTS, row = u / PARTS;  // (sequence, token, head)
    const int Hkv = static_cast<int>(cut.heads.d), lp = cut.lp;
    const int tok = fdiv(row, cut.heads), g = row - tok * Hkv;
    const int b = fdiv(tok, cut.chunk), i = tok - b * a.chunk;
    const int p = a.hist + i, j = 8 * part;
    const size_t src = static_cast<size_t>(row) * D + j;
    const size_t slot = (static_cast<size_t>(b) * Hkv + g) * lp + p;
    const size_t prow = (static_cast<size_t>(b) * Hkv + g) * plain.rows + p;
    uint4 ka = *reinterpret_cast<const uint4*>(a.k + src), kb = *reinterpret_cast<const uint4*>(a.k + src + D / 2);
    const uint4 va = *reinterpret_cast<const uint4*>(a.v + src), vb = *reinterpret_cast<const uint4*>(a.v + src + D / 2);
    const float4* ct = reinterpret_cast<const float4*>(cos_tab + static_cast<size_t>(p) * (D / 2) + j);
    const float4* st = reinterpret_cast<const float4*>(sin_tab + static_cast<size_t>(p) * (D / 2) + j);
    const float4 c0 = ct[0], c1 = ct[1], s0 = st[0], s1 = st[1];
    turn(ka.x, kb.x, c0.x, c0.y, s0.x, s0.y);
    turn(ka.y, kb.y, c0.z, c0.w, s0.z, s0.w);
    turn(ka.z, kb.z, c1.x, c1.y, s1.x, s1.y);
    turn(ka.w, kb.w, c1.z, c1.w, s1.z, s1.w);
    uint8_t* kc = c.k_codes + slot * (D / 2);
    uint8_t* vc = c.v_codes + slot * (D / 2);
    uint16_t* ks = c.k_scales + slot * (D / kKv4Group);
    uint16_t* vs = c.v_scales + slot * (D / kKv4Group);
    uint16_t* ko = plain.k == nullptr ? nullptr : plain.k + prow * D;
    uint16_t* vo = plain.v == nullptr ? nullptr : plain.v + prow * D;
    put(ka, j, mine, kc, ks, ko);
    put(kb, j + D / 2, mine, kc, ks, ko);
    put(va, j, mine, vc, vs, vo);
    put(vb, j + D / 2, mine, vc, vs, vo);
}

// One CTA reads kReadWords words of 8 values, of k or of v, of consecutive slots of a head, kReadEach per
// thread, all of whose loads are in flight together.
constexpr int kReadEach = 8, kReadWords = kThreads * kReadEach;
struct ReadCut {
    FastDiv parts;  // CTAs per head and array
    int first, count, lp;
};
template <int D>
ReadCut read_cut(int first, int count, int lp) {
    return {make_fastdiv(static_cast<int>((static_cast<long long>(count) * (D / 8) + kReadWords - 1) / kReadWords)), first,
            count, lp};
}

template <int D>
__device__ __forceinline__ void read_part(int block, const ReadCut& r, const Kv4Cache& c, const Kv4Plain& plain) {
    constexpr int WORDS = D / 8;
    const bool v = block & 1;
    const int head = fdiv(block >> 1, r.parts), part = (block >> 1) - head * static_cast<int>(r.parts.d);
    const size_t slot = static_cast<size_t>(head) * r.lp + r.first;
    const uint32_t* codes = reinterpret_cast<const uint32_t*>((v ? c.v_codes : c.k_codes) + slot * (D / 2));
    const uint16_t* scales = (v ? c.v_scales : c.k_scales) + slot * (D / kKv4Group);
    uint4* out = reinterpret_cast<uint4*>((v ? plain.v : plain.k) + static_cast<size_t>(head) * plain.rows * D);
    const int last = r.count * WORDS;  // count is at most 2^20
    uint32_t w[kReadEach], m[kReadEach];
    const int u0 = part * kReadWords + static_cast<int>(threadIdx.x);
#pragma unroll
    for (int i = 0; i < kReadEach; ++i) {
        const int u = u0 + i * kThreads;
        if (u < last) {
            w[i] = codes[u];
            m[i] = scales[u / 4];
        }
    }
#pragma unroll
    for (int i = 0; i < kReadEach; ++i) {
        const int u = u0 + i * kThreads;
        if (u < last) {
            uint32_t x[4];
            kv4_values(w[i], m[i], x);
            out[u] = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(Kv4New a, AppendCut cut, const float* __restrict__ cos_tab,
                                                              const float* __restrict__ sin_tab, Kv4Cache c, Kv4Plain plain,
                                                              ReadCut history) {
    // A dependent launch: it reads and writes only after the stream's previous kernel, and the kernel after it
    // (flash_fwd, whose prologue reads q) may be resident by then.
    griddep_wait();
    griddep_launch_dependents();
    const int block = static_cast<int>(blockIdx.x);
    if (block < cut.blocks)
        append_unit<D>(block * kThreads + static_cast<int>(threadIdx.x), a, cut, cos_tab, sin_tab, c, plain);
    else  // the history in front of the chunk, to the workspace
        read_part<D>(block - cut.blocks, history, c, plain);
}

template <int D>
__global__ void __launch_bounds__(kThreads) kv4_read_kernel(ReadCut cut, Kv4Cache c, Kv4Plain plain) {
    griddep_wait();
    griddep_launch_dependents();
    read_part<D>(static_cast<int>(blockIdx.x), cut, c, plain);
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

}  // namespace

cudaError_t launch_kv4_append(const Shape& s, const Kv4New& a, const float* cos_tab, const float* sin_tab, const Kv4Cache& c,
                              const Kv4Plain& plain, cudaStream_t st) {
    const bool d128 = s.head_dim == 128;
    const long long units = kv4_append_units(s, a.batch, a.chunk);
    if (units > INT32_MAX - kThreads) return cudaErrorInvalidConfiguration;
    const int lp = kv4_slots(s.max_len);
    const AppendCut cut{make_fastdiv(s.n_kv_heads), make_fastdiv(a.chunk), static_cast<int>(units), lp,
                        static_cast<int>((units + kThreads - 1) / kThreads)};
    const int hist = std::max(a.hist, 1);
    const ReadCut history = d128 ? read_cut<128>(0, hist, lp) : read_cut<64>(0, hist, lp);
    const long long read =
        plain.k == nullptr || a.hist == 0 ? 0 : 2LL * a.batch * s.n_kv_heads * static_cast<long long>(history.parts.d);
    if (cut.blocks + read > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(cut.blocks + read, st, &attr);
    return cudaLaunchKernelEx(&cfg, d128 ? kv4_append_kernel<128> : kv4_append_kernel<64>, a, cut, cos_tab, sin_tab, c, plain,
                              history);
}

cudaError_t launch_kv4_read(const Shape& s, int first, int count, const Kv4Cache& c, const Kv4Plain& plain,
                            cudaStream_t st) {
    const int lp = kv4_slots(s.max_len);
    const ReadCut cut = s.head_dim == 128 ? read_cut<128>(first, count, lp) : read_cut<64>(first, count, lp);
    const long long blocks = 2LL * s.batch * s.n_kv_heads * static_cast<long long>(cut.parts.d);
    if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = dependent(blocks, st, &attr);
    return cudaLaunchKernelEx(&cfg, s.head_dim == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>, cut, c, plain);
}

}  // namespace attn
