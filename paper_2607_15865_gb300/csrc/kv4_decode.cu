// kv4_decode.cu -- decode attention over a 4-bit KV cache (format: kv4.cuh) on the tensor cores, with the
// append of the new tokens and the merge of the splits fused in.
//
// A (sequence, kv head) has G query heads x ntok new tokens = columns, taken 16 at a time (an item).
// An item's slots are cut into blocks of 32 (head_dim 128) or 64 slots; the blocks of all items, in order, are
// cut into equal runs, one per CTA, whatever the lengths (they are read on the device), so that mixed lengths load
// the SMs evenly.  Within a CTA the warps take its blocks in turn, each through a private ring of bulk
// copies with one mbarrier per stage and with its own running maximum, sum and accumulators; they meet
// once per item, in shared memory.  An item that several CTAs share is merged by the last of them to finish.
//
// Per 16 slots, with mma.sync m16n8k16 (A from registers: a tcgen05 operand would have to be written
// back to shared or tensor memory at four times the packed bytes, for products 8 or 16 columns wide):
//   S [16 cols x 16 slots]  = Q [16 x D] K^T         B fragments: a lane's 16 bytes of a slot's codes
//   O^T [D x cols]         += V^T [D x 16] P^T       A fragments: 8 bytes of four slots; P^T is S's layout
// Decoding is a shift and a masked OR of the pair (128 + c, 128 + c').  For k one fma with (s, -128 s) then
// gives c s exactly (kv4.cuh), and the zero points go as a product of their own, one further mma:
//   S -= sum over groups of (z s) (sum of q over the group), those sums in three bf16 parts.
// For v it is the difference with 128 + z and the product with s, both exact: a v that is small
// beside its group must not be what is left of two larger sums.  A row of ones in place of V^T gives the
// softmax sum, of the same rounded P that weighs V.
// The running maximum moves lazily: only when a score passes it by 2^8 are O and the sum rescaled.
//
// The new tokens: the warp that holds the block of their slots rotates, quantises and writes them, to the
// cache and to its copy of the block.  Slots past the last one are masked by position and by a scale of 0;
// a NaN group of a new token's v counts from that token on, so its scale is taken as 0 too and the
// columns that see it are set to NaN when they are written.
// Every wait is bounded: on expiry a warp records kDevErrTimeout, issues and computes nothing more, lets its
// copies land and takes part in the barriers and counts.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv4.cuh"
#include "sm100_ptx.cuh"

namespace attn {
namespace {

constexpr int kMaxSeqs = 1024;  // sequences of one launch (their block counts are summed in shared memory)
constexpr int kNone = 1 << 20;  // no new token with a NaN group

template <int D_, int NT_>
struct Cfg {
    static constexpr int D = D_, NT = NT_;       // NT: tiles of 8 columns
    static constexpr int W = NT == 1 ? 16 : 12;  // warps: what the registers allow
    static constexpr int THREADS = 32 * W;
    static constexpr int KB = 32 * 128 / D;      // slots per block
    static constexpr int ROW = D / 2;            // bytes of a slot's codes
    static constexpr int GR = D / kKv4Group;     // groups
    static constexpr int CODES = KB * ROW;       // 2048
    static constexpr int SCALES = KB * GR * 2;   // 256
    static constexpr int STAGE = 2 * (CODES + SCALES);
    static constexpr int STAGES = 2;
    static constexpr int COLS = 8 * NT;
    static constexpr int QS = D + 8;             // row stride of q in shared memory (bf16)
    static constexpr int OS = D + 4;             // row stride of a warp's O (floats)
    static constexpr int OFF_O = W * STAGES * STAGE;            // float [W][COLS][OS]
    static constexpr int OFF_ML = OFF_O + W * COLS * OS * 4;    // float [W][COLS][2]
    static constexpr int OFF_Q = OFF_ML + W * COLS * 8;         // bf16 [16][QS]
    static constexpr int OFF_PRE = OFF_Q + 16 * QS * 2;         // int [kMaxSeqs + 1]
    static constexpr int OFF_BAR = (OFF_PRE + (kMaxSeqs + 1) * 4 + 7) & ~7;
    static constexpr int OFF_NAN = OFF_BAR + W * STAGES * 8;    // int [4]: first new token with a NaN group of v
    static constexpr int OFF_FLAG = OFF_NAN + 16;
    static constexpr int BYTES = OFF_FLAG + 16;
    static_assert(CODES == 2048 && SCALES == 256 && BYTES <= 232448, "shared memory");
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
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
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

constexpr uint32_t kOnes = 0x3F803F80u, kMinus128 = 0xC300C300u;

// The scales of a pair of values: s and -128 s (for decode2), and z s.
struct Pair {
    uint32_t s, n;
};
__device__ __forceinline__ Pair pair_of(uint32_t m2, uint32_t& zs) {
    Pair p;
    p.s = m2 & 0x7FF07FF0u;
    p.n = mul2(p.s, kMinus128);
    zs = fma2((m2 & 0x000F000Fu) | 0x43004300u, p.s, p.n);
    return p;
}
struct ZPair {  // the scales s of a pair and 128 + z
    uint32_t s, z;
};
__device__ __forceinline__ ZPair zpair_of(uint32_t m2) {
    return {m2 & 0x7FF07FF0u, (m2 & 0x000F000Fu) | 0x43004300u};
}
__device__ __forceinline__ uint32_t value2(uint32_t w, int i, const ZPair& p) {
    return mul2(sub2(((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u, p.z), p.s);
}
// Pair i of a word: the two codes at bit 4 i of its halves, times s.
__device__ __forceinline__ uint32_t decode2(uint32_t w, int i, const Pair& p) {
    return fma2(((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u, p.s, p.n);
}

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a) : "memory");
    return v;
}
template <int N>
__device__ __forceinline__ void lds(uint32_t a, uint32_t (&v)[N]) {
    static_assert(N == 1 || N == 2 || N == 4, "words");
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                     : "r"(a)
                     : "memory");
    else if constexpr (N == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(a) : "memory");
    else
        v[0] = lds32(a);
}

struct Args {
    const uint16_t* q;
    const uint16_t* k_new;
    const uint16_t* v_new;
    const int32_t* d_hist;
    Kv4Cache c;
    const float* cos_tab;
    const float* sin_tab;
    uint16_t* out;
    float* part_o;   // [2 per CTA][16][D]
    float* part_ml;  // [2 per CTA][16][2]
    int* part_nan;   // [2 per CTA][4]
    int* counters;   // per item, zero between launches
    int* err;
    uint64_t wait_ns;
    float scale_log2;
    int batch, ntok, Hq, Hkv, max_len, lp, ncg, min_blocks;
};

// One warp: quantise the E values x that each lane holds of a row of D = 32 E, write the row's codes and
// scales to the cache and to the block's copy in shared memory.  Returns whether the lane's group is NaN.
template <int D>
__device__ __forceinline__ bool put_row(const float (&x)[D / 32], int lane, uint8_t* codes, uint16_t* scales,
                                        uint8_t* s_codes, uint16_t* s_scales) {
    constexpr int E = D / 32, LANES = kKv4Group / E, WL = 8 / E;  // lanes of a group and of a word
    float lo = 0.f, hi = 0.f;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        odd |= (__float_as_uint(x[e]) & 0x7F800000u) == 0x7F800000u;
    }
#pragma unroll
    for (int mask = 1; mask < LANES; mask <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, mask));
        hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, mask));
    }
    const uint32_t odds = __ballot_sync(0xFFFFFFFFu, odd);
    const bool nan = ((odds >> (lane & ~(LANES - 1))) & ((1u << LANES) - 1u)) != 0;
    const uint32_t s = kv4_scale_of(lo, hi);
    const float inv = __frcp_rn(__uint_as_float(s << 16));
    const int z = kv4_round(-lo, inv);
    const uint32_t scale = nan ? kKv4NanScale : s | static_cast<uint32_t>(z);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int j = (lane * E + e) & 7;
        const int c = min(max(kv4_round(x[e], inv) + z, 0), 15);
        w |= static_cast<uint32_t>(c) << (4 * (j >> 1) + 16 * (j & 1));
    }
    if (nan) w = 0;
#pragma unroll
    for (int mask = 1; mask < WL; mask <<= 1) w |= __shfl_xor_sync(0xFFFFFFFFu, w, mask);
    if ((lane & (WL - 1)) == 0) {
        reinterpret_cast<uint32_t*>(codes)[lane / WL] = w;
        reinterpret_cast<uint32_t*>(s_codes)[lane / WL] = w;
    }
    if ((lane & (LANES - 1)) == 0) {
        scales[lane / LANES] = static_cast<uint16_t>(scale);
        s_scales[lane / LANES] = static_cast<uint16_t>(scale);
    }
    return nan;
}

template <int E>
__device__ __forceinline__ void load_row(const uint16_t* p, int lane, float (&x)[E]) {
    if constexpr (E == 4) {
        const uint2 w = *reinterpret_cast<const uint2*>(p + 4 * lane);
        x[0] = __uint_as_float(w.x << 16);
        x[1] = __uint_as_float(w.x & 0xFFFF0000u);
        x[2] = __uint_as_float(w.y << 16);
        x[3] = __uint_as_float(w.y & 0xFFFF0000u);
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(p + 2 * lane);
        x[0] = __uint_as_float(w << 16);
        x[1] = __uint_as_float(w & 0xFFFF0000u);
    }
}

__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

template <int D, int NT>
__global__ void __launch_bounds__(Cfg<D, NT>::THREADS, 1) kv4_decode_kernel(const __grid_constant__ Args a) {
    using C = Cfg<D, NT>;
    constexpr int W = C::W, KB = C::KB, GR = C::GR, E = D / 32;
    constexpr int KW = D / 32;   // words of a lane's part of a k row (D / 4 values)
    constexpr int VW = D / 64;   // words of a lane's part of a v row (D / 8 values)
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    int* pre = reinterpret_cast<int*>(smem + C::OFF_PRE);
    int* s_nan = reinterpret_cast<int*>(smem + C::OFF_NAN);
    int* flag = reinterpret_cast<int*>(smem + C::OFF_FLAG);
    uint16_t* s_q = reinterpret_cast<uint16_t*>(smem + C::OFF_Q);
    float* s_o = reinterpret_cast<float*>(smem + C::OFF_O);
    float* s_ml = reinterpret_cast<float*>(smem + C::OFF_ML);
    auto bar = [&](int stage) { return base + C::OFF_BAR + 8u * static_cast<uint32_t>(warp * C::STAGES + stage); };
    auto stage_at = [&](int stage) { return static_cast<uint32_t>((warp * C::STAGES + stage) * C::STAGE); };
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < C::STAGES; ++s) mbar_init(bar(s), 1);
        fence_mbar_init();
    }
    griddep_wait();
    griddep_launch_dependents();

    // blocks of each sequence, and their running sums.  The blocks of a launch are counted in int: a cache of 2^31
    // of them would take 2^31 x 4.5 KB / 16 column groups.
    for (int b = tid; b < a.batch; b += C::THREADS) {
        const int h = a.d_hist[b];
        const bool ok = h >= 0 && h <= a.max_len - a.ntok;
        if (!ok && blockIdx.x == 0) atomicOr(a.err, kDevErrHistRange);
        pre[b + 1] = ok ? (h + a.ntok + KB - 1) / KB : 0;
    }
    __syncthreads();
    if (warp == 0) {
        int sum = 0;
        for (int b0 = 0; b0 < a.batch; b0 += 32) {
            int v = b0 + lane < a.batch ? pre[b0 + lane + 1] : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
                if (lane >= d) v += u;
            }
            if (b0 + lane < a.batch) pre[b0 + lane + 1] = sum + v;
            sum += __shfl_sync(0xFFFFFFFFu, v, 31);
        }
        if (lane == 0) pre[0] = 0;
    }
    __syncthreads();
    const int hc = a.Hkv * a.ncg;  // items of a sequence
    const int total = pre[a.batch] * hc;
    const int nc = min(static_cast<int>(gridDim.x), max(1, (total + a.min_blocks - 1) / a.min_blocks));
    const int cta = static_cast<int>(blockIdx.x);
    if (total == 0 || cta >= nc) return;
    auto start = [&](int j) { return static_cast<int>(static_cast<long long>(total) * j / nc); };
    auto cta_of = [&](int r) { return static_cast<int>((static_cast<long long>(r + 1) * nc - 1) / total); };
    const int r0 = start(cta), r1 = start(cta + 1);

    // where block r lies: sequence, item of the sequence, block of the item
    auto find = [&](int r, int& b) {
        while (r >= pre[b + 1] * hc) ++b;
    };
    int b_first = 0;
    {
        int hi = a.batch - 1;  // the first sequence that ends past r0
        while (b_first < hi) {
            const int mid = (b_first + hi) >> 1;
            if (pre[mid + 1] * hc > r0) hi = mid;
            else b_first = mid + 1;
        }
    }

    // the warp's blocks: r0 + warp, + W, ...; copies run up to STAGES blocks ahead
    int next = r0 + warp, b_next = b_first;
    uint32_t issued = 0;
    bool dead = false;
    auto issue = [&]() {
        if (next >= r1 || dead) return;
        find(next, b_next);
        const int rem = next - pre[b_next] * hc, T = pre[b_next + 1] - pre[b_next];
        const int blk = rem % T, head = rem / T / a.ncg;
        if (lane == 0) {
            const int st = static_cast<int>(issued % C::STAGES);
            const size_t slot = (static_cast<size_t>(b_next) * a.Hkv + head) * a.lp + static_cast<size_t>(blk) * KB;
            const uint32_t dst = base + stage_at(st);
            mbar_arrive_expect_tx(bar(st), C::STAGE);
            bulk_g2s(dst, a.c.k_codes + slot * C::ROW, C::CODES, bar(st));
            bulk_g2s(dst + C::CODES, a.c.v_codes + slot * C::ROW, C::CODES, bar(st));
            bulk_g2s(dst + 2 * C::CODES, a.c.k_scales + slot * GR, C::SCALES, bar(st));
            bulk_g2s(dst + 2 * C::CODES + C::SCALES, a.c.v_scales + slot * GR, C::SCALES, bar(st));
        }
        ++issued;
        next += W;
    };
    __syncwarp();
#pragma unroll
    for (int s = 0; s < C::STAGES; ++s) issue();

    uint32_t done = 0;
    int b_seg = b_first;
    for (int seg = r0; seg < r1;) {
        // the item of block `seg`, up to where it or the CTA's run ends
        find(seg, b_seg);
        const int b = b_seg, T = pre[b + 1] - pre[b];
        const int rem = seg - pre[b] * hc, item = rem / T, head = item / a.ncg, cg = item % a.ncg;
        const int i0 = pre[b] * hc + item * T;  // the item's first block
        const int end = min(r1, i0 + T);
        const int hist = a.d_hist[b], G = a.Hq / a.Hkv;
        const int c0 = cg * 16, ncol = min(16, G * a.ntok - c0);
        auto token = [&](int col) { return (c0 + col) / G; };
        auto row_of = [&](int col) {  // of q and out, in rows of D
            return (static_cast<size_t>(b) * a.ntok + token(col)) * a.Hq + head * G + (c0 + col) % G;
        };
        // q of the columns, rotated and rounded to bf16; columns that do not exist are 0
        for (int u = tid; u < 16 * (D / 2); u += C::THREADS) {
            const int col = u / (D / 2), j = u % (D / 2);
            uint16_t lo = 0, hi = 0;
            if (col < ncol) {
                const uint16_t* src = a.q + row_of(col) * D;
                const size_t p = static_cast<size_t>(hist + token(col)) * (D / 2) + j;
                const float x = __uint_as_float(static_cast<uint32_t>(src[j]) << 16);
                const float y = __uint_as_float(static_cast<uint32_t>(src[j + D / 2]) << 16);
                const float cs = a.cos_tab[p], sn = a.sin_tab[p];
                lo = __bfloat16_as_ushort(__float2bfloat16_rn(__fsub_rn(__fmul_rn(x, cs), __fmul_rn(y, sn))));
                hi = __bfloat16_as_ushort(__float2bfloat16_rn(__fadd_rn(__fmul_rn(y, cs), __fmul_rn(x, sn))));
            }
            s_q[col * C::QS + j] = lo;
            s_q[col * C::QS + j + D / 2] = hi;
        }
        if (tid < 4) s_nan[tid] = kNone;
        __syncthreads();

        // Q's A fragments: lane (g, t) holds values D/4 t .. D/4 t + D/4 - 1 of columns g (and g + 8); step (w, h)
        // of the products takes values 8 w + 4 h .. + 3 of them.  qz: minus their sum in three parts.
        uint32_t qa[NT][2 * KW][2], qz[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t row = base + C::OFF_Q + ((g + 8 * n) * C::QS + (D / 4) * t) * 2;
            float total_q = 0.f;
#pragma unroll
            for (int s = 0; s < 2 * KW; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w = lds32(row + 8 * s + 4 * e);
                    qa[n][s][e] = w;
                    total_q += __uint_as_float(w << 16) + __uint_as_float(w & 0xFFFF0000u);
                }
            const float p0 = round_bf16(-total_q), p1 = round_bf16(-total_q - p0), p2 = (-total_q - p0) - p1;
            qz[n][0] = pack2(p0, p1);
            qz[n][1] = pack2(p2, 0.f);
        }
        float o[NT][4 * VW][4] = {}, sum[NT][4] = {};  // sum: rows 8 .. 15 the softmax sum
        float m[NT], ml[NT];                          // running maximum of the column (scaled by log2 e / sqrt D)
        int lim[NT];                                  // last slot that the column sees
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = -INFINITY;
            ml[n] = 0.f;  // m, or 0 while that is -inf
            lim[n] = hist + (g + 8 * n < ncol ? token(g + 8 * n) : a.ntok - 1);
        }

        for (int r = r0 + warp + static_cast<int>(done) * W; r < end; r += W) {
            const int st = static_cast<int>(done % C::STAGES);
            const int k0 = (r - i0) * KB;
            if (!dead && !mbar_wait(bar(st), (done / C::STAGES) & 1u, nullptr, a.wait_ns)) {
                dead = true;
                if (lane == 0) record_dev_err(a.err, kDevErrTimeout);
            }
            ++done;
            dead = __any_sync(0xFFFFFFFFu, dead);
            if (dead) continue;
            const uint32_t s_k = base + stage_at(st), s_v = s_k + C::CODES, s_ks = s_v + C::CODES, s_vs = s_ks + C::SCALES;
            const bool tail = k0 + KB > hist;  // the block holds slots of new tokens, or none at all
            if (tail) {
                const int lo = max(k0, hist), hi = min(k0 + KB, hist + a.ntok);
                uint8_t* gs = smem + stage_at(st);
                for (int p = lo; p < hi; ++p) {
                    const size_t src = ((static_cast<size_t>(b) * a.ntok + (p - hist)) * a.Hkv + head) * D;
                    const size_t slot = (static_cast<size_t>(b) * a.Hkv + head) * a.lp + p;
                    float x[E], y[E], v[E];
                    load_row<E>(a.k_new + src, lane, x);
                    load_row<E>(a.v_new + src, lane, v);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const size_t j = static_cast<size_t>(p) * (D / 2) + (lane & 15) * E + e;
                        const float other = __shfl_xor_sync(0xFFFFFFFFu, x[e], 16), cs = a.cos_tab[j], sn = a.sin_tab[j];
                        y[e] = round_bf16(lane < 16 ? __fsub_rn(__fmul_rn(x[e], cs), __fmul_rn(other, sn))
                                                    : __fadd_rn(__fmul_rn(x[e], cs), __fmul_rn(other, sn)));
                    }
                    const int i = p - k0;
                    put_row<D>(y, lane, a.c.k_codes + slot * C::ROW, a.c.k_scales + slot * GR, gs + i * C::ROW,
                               reinterpret_cast<uint16_t*>(gs + 2 * C::CODES) + i * GR);
                    const bool nan = put_row<D>(v, lane, a.c.v_codes + slot * C::ROW, a.c.v_scales + slot * GR,
                                                gs + C::CODES + i * C::ROW,
                                                reinterpret_cast<uint16_t*>(gs + 2 * C::CODES + C::SCALES) + i * GR);
                    if (nan && lane % (kKv4Group / E) == 0) atomicMin(&s_nan[lane / (kKv4Group / E)], p - hist);
                }
                __syncwarp();
            }
            const int last = hist + a.ntok - 1 - k0;  // last slot of the block that holds a token
#pragma unroll
            for (int half = 0; half < KB / 32; ++half) {
                if (half > 0 && 32 * half > last) break;
                // scores of 32 slots: lane (g, t) has columns g, g + 8 at slots 2 t, 2 t + 1 of each 8
                float s[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = 32 * half + 8 * j + g;
                    uint32_t w[KW], zs;
                    lds<KW>(s_k + key * C::ROW + t * (KW * 4), w);
                    const uint32_t sc = lds16(s_ks + (key * GR + t * GR / 4) * 2);
                    const Pair p = pair_of(sc * 0x10001u, zs);
                    s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                    mma(s[j], qz[0][0], NT == 2 ? qz[NT - 1][0] : 0u, qz[0][1], NT == 2 ? qz[NT - 1][1] : 0u, zs, zs);
#pragma unroll
                    for (int e = 0; e < 2 * KW; ++e)
                        mma(s[j], qa[0][e][0], NT == 2 ? qa[NT - 1][e][0] : 0u, qa[0][e][1], NT == 2 ? qa[NT - 1][e][1] : 0u,
                            decode2(w[e / 2], 2 * (e % 2), p), decode2(w[e / 2], 2 * (e % 2) + 1, p));
                }
                bool moves = false;
                float mx[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mx[n] = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float& x = s[j][2 * n + e];
                            x *= a.scale_log2;
                            if (tail && k0 + 32 * half + 8 * j + 2 * t + e > lim[n]) x = -INFINITY;
                            mx[n] = fmaxf(mx[n], x);
                        }
                    moves |= mx[n] > m[n] + 8.f;
                }
                if (__any_sync(0xFFFFFFFFu, moves)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float x = fmaxf(mx[n], __shfl_xor_sync(0xFFFFFFFFu, mx[n], 1));
                        x = fmaxf(fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2)), m[n]);
                        const float f = m[n] == x ? 1.f : exp2_fast(m[n] - x);
                        m[n] = x;
                        ml[n] = x == -INFINITY ? 0.f : x;
                        const float f0 = __shfl_sync(0xFFFFFFFFu, f, 8 * t), f1 = __shfl_sync(0xFFFFFFFFu, f, 8 * t + 4);
#pragma unroll
                        for (int i = 0; i <= 4 * VW; ++i) {
                            float(&acc)[4] = i == 4 * VW ? sum[n] : o[n][i < 4 * VW ? i : 0];
                            acc[0] *= f0;
                            acc[1] *= f1;
                            acc[2] *= f0;
                            acc[3] *= f1;
                        }
                    }
                }
                uint32_t pb[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        pb[n][j] = pack2(exp2_fast(s[j][2 * n] - ml[n]), exp2_fast(s[j][2 * n + 1] - ml[n]));
#pragma unroll
                for (int k = 0; k < 2; ++k) {  // 16 slots
                    const int key = 32 * half + 16 * k + 2 * t;
                    uint32_t w[4][VW], sc[4];  // slots 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = key + (e & 1) + 8 * (e >> 1);
                        lds<VW>(s_v + row * C::ROW + g * (VW * 4), w[e]);
                        sc[e] = lds16(s_vs + (row * GR + g * GR / 8) * 2);
                        if (tail && (row > last || (sc[e] == kKv4NanScale && k0 + row > hist))) sc[e] = 0;
                    }
                    const ZPair p01 = zpair_of(sc[0] | (sc[1] << 16)), p23 = zpair_of(sc[2] | (sc[3] << 16));
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma(sum[n], 0u, kOnes, 0u, kOnes, pb[n][2 * k], pb[n][2 * k + 1]);
#pragma unroll
                    for (int v = 0; v < VW; ++v) {
                        const uint32_t a01 = __byte_perm(w[0][v], w[1][v], 0x5410), b01 = __byte_perm(w[0][v], w[1][v], 0x7632);
                        const uint32_t a23 = __byte_perm(w[2][v], w[3][v], 0x5410), b23 = __byte_perm(w[2][v], w[3][v], 0x7632);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t x0 = value2(a01, i, p01), x1 = value2(b01, i, p01), x2 = value2(a23, i, p23),
                                           x3 = value2(b23, i, p23);
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma(o[n][4 * v + i], x0, x1, x2, x3, pb[n][2 * k], pb[n][2 * k + 1]);
                        }
                    }
                }
            }
            if (tail) fence_proxy_async_smem();  // this warp wrote to the stage that the next copy fills
            __syncwarp();
            issue();
        }

        // The warps' parts meet.  Lane (g, t) holds columns 2 t, 2 t + 1 (+ 8 n) of values D/8 g .. D/8 g + D/8 - 1
        // and m of column g.
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float m0 = __shfl_sync(0xFFFFFFFFu, m[n], 8 * t), m1 = __shfl_sync(0xFFFFFFFFu, m[n], 8 * t + 4);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = warp * C::COLS + 8 * n + 2 * t + e;
                float* dst = s_o + col * C::OS + (D / 8) * g;
#pragma unroll
                for (int i = 0; i < 4 * VW; ++i)
                    *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[n][i][e], o[n][i][2 + e]);
                if (g == 0) {
                    s_ml[2 * col] = e ? m1 : m0;
                    s_ml[2 * col + 1] = sum[n][2 + e];
                }
            }
        }
        __syncthreads();
        const int j0 = cta_of(i0), j1 = cta_of(i0 + T - 1);  // the CTAs that share the item
        const int part = 2 * cta + (i0 >= r0 ? 1 : 0);
        for (int u = tid; u < ncol * D; u += C::THREADS) {
            const int col = u / D, d = u % D;
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < W; ++w) mx = fmaxf(mx, s_ml[2 * (w * C::COLS + col)]);
            const float mu = mx == -INFINITY ? 0.f : mx;
            float acc = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = exp2_fast(s_ml[2 * (w * C::COLS + col)] - mu);
                l += f * s_ml[2 * (w * C::COLS + col) + 1];
                acc += f * s_o[(w * C::COLS + col) * C::OS + d];
            }
            if (j0 == j1) {
                const bool nan = s_nan[d / kKv4Group] <= token(col) && s_nan[d / kKv4Group] > 0;
                a.out[row_of(col) * D + d] = nan ? 0x7FC0 : __bfloat16_as_ushort(__float2bfloat16_rn(acc / l));
            } else {
                a.part_o[(static_cast<size_t>(part) * 16 + col) * D + d] = acc;
                if (d == 0) {
                    a.part_ml[2 * (part * 16 + col)] = mx;
                    a.part_ml[2 * (part * 16 + col) + 1] = l;
                }
            }
        }
        if (j0 != j1) {
            if (tid < 4) a.part_nan[4 * part + tid] = s_nan[tid];
            __threadfence();
            __syncthreads();
            int* count = a.counters + static_cast<size_t>(b) * hc + item;
            if (tid == 0) *flag = atomicAdd(count, 1) == j1 - j0;
            __syncthreads();
            if (*flag) {  // the last of the item's CTAs merges them, in order
                __threadfence();
                if (tid == 0) *count = 0;
                auto part_of = [&](int j) { return 2 * j + (j == j0 ? 1 : 0); };
                for (int u = tid; u < ncol * D; u += C::THREADS) {
                    const int col = u / D, d = u % D;
                    float mx = -INFINITY;
                    int nan = kNone;
                    for (int j = j0; j <= j1; ++j) {
                        mx = fmaxf(mx, __ldcg(a.part_ml + 2 * (part_of(j) * 16 + col)));
                        const int first = __ldcg(a.part_nan + 4 * part_of(j) + d / kKv4Group);
                        nan = min(nan, first);
                    }
                    const float mu = mx == -INFINITY ? 0.f : mx;
                    float acc = 0.f, l = 0.f;
                    for (int j = j0; j <= j1; ++j) {
                        const int row = part_of(j) * 16 + col;
                        const float f = exp2_fast(__ldcg(a.part_ml + 2 * row) - mu);
                        l += f * __ldcg(a.part_ml + 2 * row + 1);
                        acc += f * __ldcg(a.part_o + static_cast<size_t>(row) * D + d);
                    }
                    a.out[row_of(col) * D + d] = nan <= token(col) && nan > 0
                                                     ? 0x7FC0
                                                     : __bfloat16_as_ushort(__float2bfloat16_rn(acc / l));
                }
            }
        }
        seg = end;
        if (seg < r1) __syncthreads();  // the merge buffers and q are written again
    }
    if (dead)  // copies still in flight land before the CTA's shared memory is given up
        for (uint32_t s = 0; s < C::STAGES; ++s) {
            const uint32_t i = issued > C::STAGES ? issued - C::STAGES + s : s;
            if (i < issued) mbar_wait(bar(static_cast<int>(i % C::STAGES)), (i / C::STAGES) & 1u, nullptr);
        }
}

template <int D, int NT>
cudaError_t launch(const Args& a, int num_sms, cudaStream_t st) {
    using C = Cfg<D, NT>;
    // a run of fewer than W blocks leaves warps idle, but spreads a short history over more SMs
    const long long most = static_cast<long long>(a.batch) * a.Hkv * a.ncg * ((a.max_len + C::KB - 1) / C::KB);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(
        std::max(1LL, std::min<long long>(num_sms, (most + a.min_blocks - 1) / a.min_blocks))));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv4_decode_kernel<D, NT>, a);
}

template <int D, int NT>
cudaError_t configure() {
    return cudaFuncSetAttribute(kv4_decode_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, NT>::BYTES);
}

}  // namespace

cudaError_t configure_kv4_decode() {
    cudaError_t e = configure<128, 1>();
    if (e == cudaSuccess) e = configure<128, 2>();
    if (e == cudaSuccess) e = configure<64, 1>();
    if (e == cudaSuccess) e = configure<64, 2>();
    return e;
}

cudaError_t launch_kv4_decode(const Shape& s, const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                              const int32_t* d_hist, int ntok, const Kv4Cache& c, const float* cos_tab,
                              const float* sin_tab, float* part_o, float* part_ml, int* counters, uint16_t* out, int* err,
                              int num_sms, cudaStream_t st, uint64_t wait_ns) {
    const int cols = s.n_q_heads / s.n_kv_heads * ntok;
    const size_t D = static_cast<size_t>(s.head_dim);
    for (int b0 = 0; b0 < s.batch; b0 += kMaxSeqs) {
        const size_t tok = static_cast<size_t>(b0) * ntok, heads = static_cast<size_t>(b0) * s.n_kv_heads;
        Args a;
        a.q = q + tok * s.n_q_heads * D;
        a.out = out + tok * s.n_q_heads * D;
        a.k_new = k_new + tok * s.n_kv_heads * D;
        a.v_new = v_new + tok * s.n_kv_heads * D;
        a.d_hist = d_hist + b0;
        a.lp = kv4_slots(s.max_len);
        const size_t slots = heads * a.lp;
        a.c = Kv4Cache{c.k_codes + slots * (D / 2), c.k_scales + slots * (D / kKv4Group), c.v_codes + slots * (D / 2),
                       c.v_scales + slots * (D / kKv4Group)};
        a.cos_tab = cos_tab;
        a.sin_tab = sin_tab;
        a.part_o = part_o;
        a.part_ml = part_ml;
        a.part_nan = reinterpret_cast<int*>(part_ml + static_cast<size_t>(num_sms) * 2 * 16 * 2);
        a.counters = counters;
        a.err = err;
        a.wait_ns = wait_ns;
        a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim)));
        a.batch = std::min(kMaxSeqs, s.batch - b0);
        a.ntok = ntok;
        a.Hq = s.n_q_heads;
        a.Hkv = s.n_kv_heads;
        a.max_len = s.max_len;
        a.ncg = (cols + 15) / 16;
        a.min_blocks = 8;
        const cudaError_t e = D == 128 ? (cols <= 8 ? launch<128, 1>(a, num_sms, st) : launch<128, 2>(a, num_sms, st))
                                       : (cols <= 8 ? launch<64, 1>(a, num_sms, st) : launch<64, 2>(a, num_sms, st));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace attn
