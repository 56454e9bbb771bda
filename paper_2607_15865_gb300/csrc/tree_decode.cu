// tree_decode.cu -- attention of a few new tokens per sequence, a chain or a tree, over the cache with an optional sliding
// window (the simple form: a warp per query row), and the accepted tokens' move to the end of the history.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "sm100_ptx.cuh"
#include "tree.cuh"

namespace attn {
namespace {

struct Args {
    const uint16_t* q;
    const uint16_t* k_new;
    const uint16_t* v_new;
    const int32_t* d_hist;  // NULL: hist
    const int32_t* parents;
    uint16_t* k_cache;
    uint16_t* v_cache;
    const float* cos_tab;
    const float* sin_tab;
    uint16_t* out;
    int* err;
    float scale_log2;
    int hist, batch, n, Hq, Hkv, max_len, window, sinks;
};

__device__ __forceinline__ float bf(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
__device__ __forceinline__ uint16_t bits(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// The kin of all tokens in shared memory; false: the sequence is skipped (and flagged).
__device__ __forceinline__ bool look(const Args& a, int b, int hist, uint64_t* kin_s) {
    __shared__ int ok_s;
    if (threadIdx.x < 32) {
        uint64_t kin[2];
        const int count = tree_kin(a.parents == nullptr ? nullptr : a.parents + static_cast<size_t>(b) * a.n, a.n, threadIdx.x, kin);
        kin_s[threadIdx.x] = kin[0];
        kin_s[threadIdx.x + 32] = kin[1];
        const bool range = hist < 0 || hist > a.max_len || hist + count > a.max_len;
        if (threadIdx.x == 0) {
            ok_s = count >= 0 && !range;
            if (count < 0 || range) atomicOr(a.err, (count < 0 ? kDevErrTree : 0) | (range ? kDevErrHistRange : 0));
        }
    }
    __syncthreads();
    return ok_s != 0;
}

template <int D>
__global__ void tree_append_kernel(const Args a) {
    __shared__ uint64_t kin_s[kMaxTree];
    const int i = blockIdx.x, b = blockIdx.y;
    const int hist = a.d_hist[b];
    if (!look(a, b, hist, kin_s) || kin_s[i] == 0) return;
    const int pos = hist + __popcll(kin_s[i]) - 1;
    for (int u = threadIdx.x; u < a.Hkv * D / 2; u += blockDim.x) {
        const int g = u / (D / 2), j = u % (D / 2);
        const size_t src = ((static_cast<size_t>(b) * a.n + i) * a.Hkv + g) * D + j;
        const size_t dst = ((static_cast<size_t>(b) * a.Hkv + g) * a.max_len + hist + i) * D + j;
        const float c = a.cos_tab[static_cast<size_t>(pos) * (D / 2) + j], s = a.sin_tab[static_cast<size_t>(pos) * (D / 2) + j];
        const float x = bf(a.k_new[src]), y = bf(a.k_new[src + D / 2]);
        a.k_cache[dst] = bits(__fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)));
        a.k_cache[dst + D / 2] = bits(__fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s)));
        a.v_cache[dst] = a.v_new[src];
        a.v_cache[dst + D / 2] = a.v_new[src + D / 2];
    }
}

// A warp per (token, query head): the keys one by one, in two passes over the visible ones.
template <int D, bool CHUNK>
__global__ void attend_kernel(const Args a) {
    constexpr int E = D / 64;
    __shared__ uint64_t kin_s[kMaxTree];
    const int i = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 31;
    const int hist = a.d_hist == nullptr ? a.hist : a.d_hist[b];
    uint64_t kin = 0;
    int depth = i;
    if constexpr (!CHUNK) {
        if (!look(a, b, hist, kin_s) || kin_s[i] == 0) return;
        kin = kin_s[i];
        depth = __popcll(kin) - 1;
    }
    const int pos = hist + depth, lo = max(0, pos - a.window + 1);
    for (int h = threadIdx.x >> 5; h < a.Hq; h += blockDim.x >> 5) {
        const int g = h / (a.Hq / a.Hkv);
        const size_t row = ((static_cast<size_t>(b) * a.n + i) * a.Hq + h) * D;
        float q[2 * E], acc[2 * E];
        for (int e = 0; e < E; ++e) {
            const int j = lane * E + e;
            const float c = a.cos_tab[static_cast<size_t>(pos) * (D / 2) + j], s = a.sin_tab[static_cast<size_t>(pos) * (D / 2) + j];
            const float x = bf(a.q[row + j]), y = bf(a.q[row + j + D / 2]);
            q[e] = round_bf16(__fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s)));
            q[E + e] = round_bf16(__fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s)));
            acc[e] = acc[E + e] = 0.f;
        }
        const uint16_t* kc = a.k_cache + (static_cast<size_t>(b) * a.Hkv + g) * a.max_len * D;
        const uint16_t* vc = a.v_cache + (static_cast<size_t>(b) * a.Hkv + g) * a.max_len * D;
        float m = -INFINITY, l = 0.f;
        auto key = [&](int s) {
            float d = 0.f;
            for (int e = 0; e < E; ++e)
                d += q[e] * bf(kc[static_cast<size_t>(s) * D + lane * E + e]) + q[E + e] * bf(kc[static_cast<size_t>(s) * D + D / 2 + lane * E + e]);
            for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xFFFFFFFFu, d, o);
            d *= a.scale_log2;
            const float mn = fmaxf(m, d), r = mn == -INFINITY ? 0.f : mn;
            const float w = fast_exp2(m - r), p = fast_exp2(d - r);
            l = l * w + p;
            for (int e = 0; e < E; ++e) {
                acc[e] = acc[e] * w + p * bf(vc[static_cast<size_t>(s) * D + lane * E + e]);
                acc[E + e] = acc[E + e] * w + p * bf(vc[static_cast<size_t>(s) * D + D / 2 + lane * E + e]);
            }
            m = mn;
        };
        const int end = CHUNK ? pos + 1 : hist;  // slots that are seen by position alone
        for (int s = 0; s < min(a.sinks, min(lo, end)); ++s) key(s);
        for (int s = lo; s < end; ++s) key(s);
        if constexpr (!CHUNK)
            for (int t = 0; t < a.n; ++t) {
                const int at = hist + __popcll(kin_s[t]) - 1;
                if ((kin >> t & 1) && (at >= lo || at < a.sinks)) key(hist + t);
            }
        for (int e = 0; e < E; ++e) {
            a.out[row + lane * E + e] = bits(acc[e] / l);
            a.out[row + D / 2 + lane * E + e] = bits(acc[E + e] / l);
        }
    }
}

// Layers whose caches one launch of tree_accept moves.
constexpr int kAcceptLayers = 128;
struct Accept {
    uint16_t* k[kAcceptLayers];
    uint16_t* v[kAcceptLayers];
    const int32_t* d_hist;
    const int32_t* parents;
    const int32_t* leaf;
    int32_t* new_len;
    int* err;
    int n, Hkv, max_len, row16;  // row16: 16-byte units of a row
};

// A block per (kv head, sequence, layer): the rows of the path that are not in place yet, k's and then v's, are loaded
// by all threads before any is stored: a slot that one row leaves may be the one that another moves to.
__global__ void __launch_bounds__(256) tree_accept_kernel(const Accept a) {
    constexpr int UNITS = 2 * kMaxTree * 16 / 256;  // 16-byte units of the most rows of k and v, per thread
    __shared__ int src_s[kMaxTree], count_s;
    const int g = blockIdx.x, b = blockIdx.y, layer = blockIdx.z;
    const int hist = a.d_hist[b];
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x, leaf = a.leaf[b];
        uint64_t kin[2];
        const int count = tree_kin(a.parents + static_cast<size_t>(b) * a.n, a.n, lane, kin);
        uint64_t path = 0;
        bool bad = count < 0 || leaf < -1 || leaf >= a.n;
        if (!bad && leaf >= 0) {
            const uint64_t k0 = shfl64(kin[0], leaf & 31), k1 = shfl64(kin[1], leaf & 31);
            path = leaf < 32 ? k0 : k1;
            bad = path == 0;
        }
        const bool range = hist < 0 || hist > a.max_len || hist + max(count, 0) > a.max_len;
        if (bad || range) path = 0;
        for (int h = 0; h < 2; ++h)
            if (path >> (lane + 32 * h) & 1) src_s[__popcll(path & ((1ull << (lane + 32 * h)) - 1))] = lane + 32 * h;
        if (lane == 0) {
            count_s = __popcll(path);
            if (g == 0 && layer == 0) {
                if (bad || range) atomicOr(a.err, (bad ? kDevErrTree : 0) | (range ? kDevErrHistRange : 0));
                if (a.new_len != nullptr) a.new_len[b] = hist + __popcll(path);
            }
        }
    }
    __syncthreads();
    const int rows = count_s, units = rows * a.row16;
    uint4* base[2] = {reinterpret_cast<uint4*>(a.k[layer]), reinterpret_cast<uint4*>(a.v[layer])};
    const size_t head = ((static_cast<size_t>(b) * a.Hkv + g) * a.max_len + hist) * a.row16;
    uint4 w[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = (i % (UNITS / 2)) * 256 + threadIdx.x;
        if (u < units) {
            const int j = u / a.row16;
            if (src_s[j] != j) w[i] = base[i / (UNITS / 2)][head + static_cast<size_t>(src_s[j]) * a.row16 + u % a.row16];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int u = (i % (UNITS / 2)) * 256 + threadIdx.x;
        if (u < units && src_s[u / a.row16] != u / a.row16) base[i / (UNITS / 2)][head + u] = w[i];
    }
}

Args args_of(const Shape& s, const TreeCall& c) {
    Args a;
    a.q = c.q;
    a.k_new = c.k;
    a.v_new = c.v;
    a.d_hist = c.d_hist;
    a.hist = c.hist;
    a.parents = c.parents;
    a.k_cache = c.k_cache;
    a.v_cache = c.v_cache;
    a.cos_tab = c.cos_tab;
    a.sin_tab = c.sin_tab;
    a.out = c.out;
    a.err = c.err;
    a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim)));
    a.batch = s.batch;
    a.n = c.n;
    a.Hq = s.n_q_heads;
    a.Hkv = s.n_kv_heads;
    a.max_len = s.max_len;
    a.window = c.window;
    a.sinks = c.sinks;
    return a;
}

}  // namespace

cudaError_t launch_tree_decode(const Shape& s, const TreeCall& c, cudaStream_t st) {
    const Args a = args_of(s, c);
    const dim3 grid(static_cast<unsigned>(c.n), static_cast<unsigned>(s.batch));
    if (c.d_hist == nullptr) {
        if (s.head_dim == 128)
            attend_kernel<128, true><<<grid, 256, 0, st>>>(a);
        else
            attend_kernel<64, true><<<grid, 256, 0, st>>>(a);
        return cudaGetLastError();
    }
    if (s.head_dim == 128) {
        tree_append_kernel<128><<<grid, 128, 0, st>>>(a);
        attend_kernel<128, false><<<grid, 256, 0, st>>>(a);
    } else {
        tree_append_kernel<64><<<grid, 128, 0, st>>>(a);
        attend_kernel<64, false><<<grid, 256, 0, st>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t launch_tree_accept(const Shape& s, const int32_t* d_hist, const int32_t* parents, const int32_t* leaf, int n,
                               uint16_t* const* k_caches, uint16_t* const* v_caches, int layers, int32_t* new_len, int* err,
                               cudaStream_t st) {
    Accept a;
    a.d_hist = d_hist;
    a.parents = parents;
    a.leaf = leaf;
    a.err = err;
    a.n = n;
    a.Hkv = s.n_kv_heads;
    a.max_len = s.max_len;
    a.row16 = s.head_dim / 8;
    for (int l0 = 0; l0 < layers; l0 += kAcceptLayers) {
        const int count = std::min(layers - l0, kAcceptLayers);
        std::copy(k_caches + l0, k_caches + l0 + count, a.k);
        std::copy(v_caches + l0, v_caches + l0 + count, a.v);
        a.new_len = l0 == 0 ? new_len : nullptr;
        const dim3 grid(static_cast<unsigned>(s.n_kv_heads), static_cast<unsigned>(s.batch), static_cast<unsigned>(count));
        tree_accept_kernel<<<grid, 256, 0, st>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace attn
