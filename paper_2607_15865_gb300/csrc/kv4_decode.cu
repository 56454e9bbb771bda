// kv4_decode.cu -- decode attention over a 4-bit KV cache (format: kv4.cuh) on the tensor cores, with the
// append of the new tokens and the merge of the splits fused in.
//
// A (sequence, kv head) has G query heads x ntok new tokens = columns, taken 16 at a time (an item).
// An item's slots are cut into blocks of 32 (head_dim 128) or 64 slots; the lengths are read on the device.
//   few items        (up to half the SMs) each item's blocks in equal pieces, one per CTA, as many as the SMs allow and
//                    in proportion to the lengths: one CTA of 12 (more than 8 columns: 8) warps per SM, so that
//                    an item has few parts to merge
//   many             the blocks of all items, in order, in equal runs, whatever the lengths: each item counts
//                    kItemCost blocks more than it has, for what it costs to begin and to end one; or in whole items,
//                    where they are short or about as many as the CTAs.  CTAs of four warps, several per SM: while
//                    one begins or ends an item the others walk (or of eight, for up to one item per SM of more
//                    than 8 columns)
// Within a CTA the warps take an item's blocks in turn, each through a private ring of two stages, filled by
// cp.async (ten 16-byte copies per lane; as four bulk copies and an mbarrier a block cost 50 instructions
// more), and with its own running maximum, sum and accumulators; they meet once per item, in shared memory.  An
// item that several CTAs share is merged by the last of them to finish, in a fixed order.
//
// Per 16 slots, with mma.sync m16n8k16 (A from registers: a tcgen05 operand would have to be written
// back to shared or tensor memory at four times the packed bytes, for products 8 or 16 columns wide):
//   S^T [16 slots x cols]   = K [16 x D] Q^T         A fragments: a lane's 16 bytes of two slots' codes
//   O^T [D x cols]         += V^T [D x 16] P^T       A fragments: 8 bytes of four slots
// P^T goes from the layout of the first's result to the operand of the second by an 8 x 8 transpose
// (movmatrix) per 8 slots.  (With S [cols x slots] it needs none, but its Q fragments are half zeros for
// up to 8 columns, and the moves that set them up cost more than the products.)
// Decoding: a code in bits 0 .. 3 of a bf16 that is otherwise 0 is the subnormal c 2^-133, and in bits 4 .. 7 it is
// 16 c 2^-133 (where the exponent's first bit comes in, the spacing is still that of the subnormals).  So one AND
// makes a pair of numbers, without a shift for every other pair, and one product with s 2^60, or s 2^56,
// makes c s 2^-73, exactly (kv4.cuh); scales of 2^-53 to 2^67 stay in the range of bf16.  Scores are in units of
// 2^-73; P and its sum are 2^60 times as large, so that small weights of small values stay above the
// least float.  For k the zero points go as a product of their own, one further mma:
//   S -= sum over groups of (z s) (sum of q over the group), those sums in three bf16 parts.
// For v it is one fma with - z s instead of the product: a v that is small beside its group must not be
// what is left of two larger sums.  At head_dim 128 rows of ones in place of V^T give the softmax sum, of the same
// rounded P that weighs V; at 64 the lanes add P up in float.
// The running maximum moves lazily: only when a score passes it by 2^8 are O and the sum rescaled.
// Roundings: q and the new k to bf16 after RoPE, as the bf16 stages round them; a weight P, as over the bf16 cache, at
// head_dim 128 to bf16 (the operand's type), and at 64, where that decode keeps it to float precision, to the sum of two
// bf16 numbers, within 2^-16; the output.  Scores, maxima, sums and O are floats.  The second number costs a further mma per
// V operand (calls in a graph, 32 / 8 heads of 64 values: 16 x 8191 25.6 us without and 27.7 with it, 64 x 8191 74.4 and
// 82.1).
//
// What bounds it: no unit's rate, but the latencies of few warps.  16 slots of a head of 128 values with up to 8 columns
// take 294 warp instructions, 18 of them mma, and 437 cycles of a scheduler, at which the SMs walk about 6 TB/s.  Over a
// whole call (16 x 8191, cold) a scheduler has 3.7 warps and issues in 58% of its cycles, the ALU pipe is at 50%, the tensor
// pipe at 24%, the DRAM at 56%; of the time from one instruction of a warp to its next, 22% goes to fixed latencies, 16% to
// the issue, 16% to other warps' turns, 12% to a busy pipe, 8% to barriers, 6% to fetching instructions, 4% to global
// memory.  The walk at its rate is 25 us of the call's 37.6; beginning and ending items is the rest.  With few items
// (4 tokens over 8188: two warps, 29%) barriers, shared memory and the fetch of instructions take 42%.  Around the walk a
// call takes 5 us for one short sequence (launch, lengths, first bytes, the warps' meeting) and about 2 us more where
// items are shared.  In a graph, 32 / 8 heads of 128 values (in brackets the bytes at 6.77 TB/s), us: 1 x 1 4.6, 1 x 1024
// 7.0 (0.2), 16 x 1024 12.8 (2.8), 16 x 8191 37.6 (22.3), 64 x 8191 119 (89.4), 4 tokens over 8188 12.5 (1.4); 40 / 8 heads
// 1 x 32767 13.9 (5.6); 32 / 8 heads of 64 1 x 1024 6.1 (0.1), 16 x 8191 27.7 (11.2), 64 x 8191 82 (44.7).  Over the bf16 cache,
// heads of 128, 1 x 1024 7.6, 16 x 8191 79, 64 x 8191 311, 1 x 32767 26.9.
//
// The new tokens: a CTA that holds their slots rotates and quantises them, a warp per row, before its own
// blocks, writes them to the cache and stages them for the warp that has their block.  Slots past the last
// one are masked by position and by a scale of 0; a group of a new token's v that is NaN, or that the products would make
// so (a scale of 2^68 or more), counts from that token on, so its scale is taken as 0 too and the columns that see it are
// set to NaN when they are written.
// The only wait on other warps that is not a barrier, for the staged rows, is bounded: on expiry the warp records
// kDevErrTimeout and the item's outputs are not written.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "kv4.cuh"
#include "sm100_ptx.cuh"

namespace attn {
namespace {

constexpr int kMaxSeqs = 128;   // sequences of one launch (their block counts are summed in shared memory)
// Blocks that it costs a CTA to begin and end an item.  Calls in a graph (32 / 8 heads of 128 values, us) with 0, 8, 16, 32:
// 16 sequences of mixed lengths 33.1, 26.6, 24.5, 25.5; of 8191 40.2, 38.4, 37.2, 38.3; of 1024 16.4, 12.7, 13.2, 14.7.
constexpr int kItemCost = 16;
// Blocks of a piece, unless the item is but one: a merge takes 2 us or more, a block of each warp 0.5.  With 16 warps, one
// sequence of 300, 500 and 700 tokens took 5.4, 6.2 and 7.1 us in one piece, 7.7, 8.1 and 8.2 in several, 1000 tokens 8.0
// in either, and 8.3 in pieces of 8 blocks at least; with 16 columns 400 tokens 8.5 and 10.4.
constexpr int kMinBlocks = 4;
constexpr int kMaxNew = 16;     // new tokens per sequence
constexpr int kNone = 1 << 20;  // no new token with a NaN group

// How the items are cut: pieces, or runs with few items or many.
enum Cut { kPieces, kRunsFew, kRuns };

template <int D_, int NT_, Cut CUT_>
struct Cfg {
    static constexpr int D = D_, NT = NT_;       // NT: tiles of 8 columns
    static constexpr bool WIDE = CUT_ == kPieces;
    static constexpr int PARTS = D == 64 ? 2 : 1;  // bf16 numbers that a weight is the sum of
    // Warps, and CTAs per SM: what registers and shared memory allow.  Pieces of 8 columns with 16, 12 and 8 warps (head_dim
    // 128, us): 1 x 2000 tokens 7.7, 7.0, 6.5, 1 x 32767 14.4, 14.5, 15.1, 4 x 8000 14.7, 14.8, 15.9; head_dim 64 with
    // 16 and 12: 1 x 1024 6.5 and 6.1, 1 x 8191 7.95 and 7.5, 1 x 30000 10.5 and 10.65, 4 x 8000 11.05 and 11.25.  Many
    // runs with 4, 3 and 2 CTAs, the last of 8 warps: 16 x 8191 37.8, 36.8, 39.3, 64 x 2000 38.2, 40.6, 43.9, 16 of mixed
    // lengths 24.6, 24.0, 26.6.
    static constexpr int W = CUT_ == kRuns ? 4 : NT == 2 ? 8 : 12;
    static constexpr int CTAS = CUT_ != kRuns ? 1 : NT == 1 ? 4 : D == 128 ? 2 : 3;
    static constexpr int THREADS = 32 * W;
    static constexpr int ALONE = NT == 1 ? 24 : 16;   // pieces: an item of up to so many blocks is one (see kMinBlocks)
    // runs: blocks that a CTA may have more than its run, where that saves all merges, and the longest item of mixed
    // ones (with figures where the runs are cut)
    static constexpr int EXCESS = NT == 1 ? 20 : CUT_ == kRunsFew ? 48 : 32;
    static constexpr int LONGEST = NT == 1 ? 36 : 48;
    // Parts that a merging thread loads at once: all of the most pieces that there are for 8 heads, if registers allow
    // (1 x 32767: 14.4 us with 8, 13.9 with 10; 4 tokens over 8188 13.5 with 10, 12.2 with 20); few runs share an item (16
    // sequences of 8 tokens over 4000 53.1 with 16, 51.9 with 4).
    static constexpr int BATCH = CUT_ == kPieces ? (NT == 1 ? 10 : 20) : NT == 1 ? 8 : 4;
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
    static constexpr int O_BYTES = COLS * OS * 4;  // of a warp
    static constexpr int NEW = ROW + 2 * GR;     // bytes of a staged row: codes, scales
    static constexpr int OFF_O = W * STAGES * STAGE;            // float [W][COLS][OS]; before that staged rows (stage_row)
    static constexpr int OFF_ML = OFF_O + W * O_BYTES;          // float [W][COLS][2]
    static constexpr int OFF_Q = OFF_ML + W * COLS * 8;         // bf16 [COLS][QS]
    static constexpr int OFF_PRE = OFF_Q + COLS * QS * 2;       // int [kMaxSeqs + 1]: blocks and costs before a sequence
    static constexpr int OFF_FREE = OFF_PRE + (kMaxSeqs + 1) * 4;  // uint8 [kMaxSeqs]: slots of the last block past the last token
    static constexpr int OFF_BAR = (OFF_FREE + kMaxSeqs + 7) & ~7;  // mbarrier: the staged rows
    static constexpr int OFF_NAN = OFF_BAR + 8;                 // int [4]: first new token with a NaN group of v
    // int [3]: whether this CTA merges its first, its last item; whether the wait for the staged rows ran out
    static constexpr int OFF_FLAG = OFF_NAN + 16;
    static constexpr int OFF_SEG = OFF_FLAG + 12;               // Segment [2]: of this turn, and a held one
    static constexpr int BYTES = OFF_SEG + 2 * 40;
    static_assert(CODES == 2048 && SCALES == 256 && NEW % 4 == 0 && 2 * kMaxNew * NEW <= O_BYTES, "layout");
    static_assert(BYTES <= 232448 && CTAS * (BYTES + 1024) <= 233472, "shared memory");
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same on zeros.
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr uint32_t kOnes = 0x3F803F80u;                       // 1
constexpr uint32_t kUp = 0x5D805D80u, kSixteenth = 0x3D803D80u;  // 2^60, 2^-4
constexpr float kUnit = 9.44473296573929e21f;                // 2^73
constexpr float kLift = 60.f;                                // P is 2^60 times the weights
constexpr uint32_t kTooLarge = 0x6180u;                      // scales from 2^68 on: times 2^60 they are infinite

// The scales of a pair of values, for codes in the low and in the high four bits of a byte, and z s (in
// units of 2^-73).
struct Pair {
    uint32_t lo, hi, zs;
};
__device__ __forceinline__ Pair pair_of(uint32_t m2) {
    Pair p;
    p.lo = mul2(m2 & 0x7FF07FF0u, kUp);
    p.hi = mul2(p.lo, kSixteenth);
    p.zs = mul2(m2 & 0x000F000Fu, p.lo);
    return p;
}
// Pair i of a word and of the same word shifted right by 8: c s, and (c - z) s with p.zs negated.
__device__ __forceinline__ uint32_t code2(uint32_t w, uint32_t w8, int i, const Pair& p) {
    const uint32_t x = i < 2 ? w : w8;
    return i % 2 == 0 ? mul2(x & 0x000F000Fu, p.lo) : mul2(x & 0x00F000F0u, p.hi);
}
__device__ __forceinline__ uint32_t value2(uint32_t w, uint32_t w8, int i, const Pair& p) {
    const uint32_t x = i < 2 ? w : w8;
    return i % 2 == 0 ? fma2(x & 0x000F000Fu, p.lo, p.zs) : fma2(x & 0x00F000F0u, p.hi, p.zs);
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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

// Adds to a counter after what this CTA wrote before its last barrier, and before what it reads after its next.
__device__ __forceinline__ int add_acq_rel(int* p, int v) {
    int old;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
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
    float scale_log2, move;  // log2 e / sqrt D in units of 2^-73, and the lead of a score that moves the maximum (2^8)
    int batch, ntok, Hq, Hkv, max_len, lp, ncg, hist;
};

// One warp: quantise the E = D / 32 values of a row that each lane holds (bf16 pairs; with E = 2 one pair), write
// the row's codes and scales to the cache and to a staged row (codes, then scales).  Returns whether the lane's
// group is NaN, or NaN to the products.
template <int D>
__device__ __forceinline__ bool put_row(const uint32_t (&x)[D / 64], int lane, uint8_t* codes, uint16_t* scales,
                                        uint8_t* staged) {
    constexpr int E = D / 32, LANES = kKv4Group / E, WL = 8 / E;  // lanes of a group and of a word
    const uint32_t all[4] = {x[0], x[E / 2 - 1], x[0], x[0]};
    uint32_t e = kv4_extremes(all);
#pragma unroll
    for (int mask = 1; mask < LANES; mask <<= 1) e = max2(e, __shfl_xor_sync(0xFFFFFFFFu, e, mask));
    float inv;
    const uint32_t scale = kv4_group(e, inv);
    const bool nan = scale == kKv4NanScale;
    const int z = static_cast<int>(scale & 15u);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i)
        w |= (kv4_code(bf_lo(x[i]), inv, z) | kv4_code(bf_hi(x[i]), inv, z) << 16) << (4 * ((lane * (E / 2) + i) & 3));
    if (nan) w = 0;
#pragma unroll
    for (int mask = 1; mask < WL; mask <<= 1) w |= __shfl_xor_sync(0xFFFFFFFFu, w, mask);
    if ((lane & (WL - 1)) == 0) {
        reinterpret_cast<uint32_t*>(codes)[lane / WL] = w;
        reinterpret_cast<uint32_t*>(staged)[lane / WL] = w;
    }
    if ((lane & (LANES - 1)) == 0) {
        scales[lane / LANES] = static_cast<uint16_t>(scale);
        reinterpret_cast<uint16_t*>(staged + D / 2)[lane / LANES] = static_cast<uint16_t>(scale);
    }
    return scale >= kTooLarge;
}

template <int N>
__device__ __forceinline__ void load_row(const uint16_t* p, int lane, uint32_t (&x)[N]) {
    if constexpr (N == 2) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(p + 4 * lane));
        x[0] = w.x;
        x[1] = w.y;
    } else {
        x[0] = __ldg(reinterpret_cast<const uint32_t*>(p + 2 * lane));
    }
}

__device__ __forceinline__ float round_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// Inclusive sum over the lanes of a warp.
__device__ __forceinline__ int warp_scan(int v, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, v, d);
        if (lane >= d) v += u;
    }
    return v;
}

// The part of an item that a CTA walks: its blocks lo .. hi - 1 of T.
struct Segment {
    int b, item, head, T, hist;
    int c0, ncol;      // the item's columns
    int lo, hi, base;  // base: the item's block 0 in the order that runs are cut from
};

// x / y for 0 <= x < 2^20, y > 0: (x + 1/2) / y is at least 1 / 2y from an integer, twice what the float quotient
// may be off by.
__device__ __forceinline__ int small_div(int x, int y) {
    return static_cast<int>(__fdividef(static_cast<float>(x) + 0.5f, static_cast<float>(y)));
}
__device__ __forceinline__ int small_ceil_div(int x, int y) { return small_div(x - 1, y) + 1; }  // x > 0

// One warp: piece `cta` where the items of up to 32 sequences are cut into pieces of at most `target` blocks, with the
// least target (of 32 tried) for which the pieces are at most per for each of the hc items of a sequence.  Lane b
// holds the blocks T of an item of sequence b (0: skipped).  The item's block 0 .. : T, hist, lo, hi; base:
// the piece, c0: the pieces of the item (0: there is no piece `cta`).
__device__ __forceinline__ Segment piece_of(int T, int hist, int hc, int per, int alone, int cta, int lane) {
    Segment w = {};
    const uint32_t live = __ballot_sync(0xFFFFFFFFu, T > 0);
    const int items = __popc(live), sum = __reduce_add_sync(0xFFFFFFFFu, T), longest = __reduce_max_sync(0xFFFFFFFFu, T);
    if (items == 0) return w;
    int target = max(kMinBlocks, small_ceil_div(longest, small_div(per, items)));  // fits
    if (longest * items != sum) {
        const int least = max(kMinBlocks, (sum + per - 1) / per);  // no less fits
        const int mine = least + (((target - least) * lane) >> 5);
        int pieces = 0;
        for (uint32_t rest = live; rest != 0; rest &= rest - 1)
            pieces += small_ceil_div(__shfl_sync(0xFFFFFFFFu, T, __ffs(rest) - 1), mine);
        const uint32_t fits = __ballot_sync(0xFFFFFFFFu, pieces <= per);
        if (fits != 0) target = __shfl_sync(0xFFFFFFFFu, mine, __ffs(fits) - 1);
    }
    const int n = T <= alone ? (T > 0 ? 1 : 0) : small_ceil_div(T, target), upto = warp_scan(n, lane);
    const uint32_t past = __ballot_sync(0xFFFFFFFFu, T > 0 && upto * hc > cta);
    if (past == 0) return w;
    w.b = __ffs(past) - 1;
    w.T = __shfl_sync(0xFFFFFFFFu, T, w.b);
    w.hist = __shfl_sync(0xFFFFFFFFu, hist, w.b);
    w.c0 = __shfl_sync(0xFFFFFFFFu, n, w.b);
    const int rem = cta - __shfl_sync(0xFFFFFFFFu, upto - n, w.b) * hc;
    w.item = small_div(rem, w.c0);
    w.base = rem - w.item * w.c0;
    const int whole = small_div(w.T, w.c0), more = w.T - whole * w.c0;
    w.lo = w.base * whole + min(w.base, more);
    w.hi = w.lo + whole + (w.base < more ? 1 : 0);
    return w;
}

// The first b with sums[b + 1] * hc > r.
__device__ __forceinline__ int search(const int* sums, int batch, int hc, int r) {
    int lo = 0, hi = batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid + 1] * hc > r) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// The maximum that a part is merged by: NaN where its sum is (then its scores may be NaN throughout, and m -inf as if
// it had none) or a score is past the largest float.  -inf: no slot of the part is seen.  inf, which mark does not return: a
// wait ran out in the part, and the item is not to be written.
__device__ __forceinline__ float mark(float m, float l) { return l != l || m == INFINITY ? NAN : m; }

// The merge of up to N parts (m, l, o[4]) with a running (m, l, o[4]); parts without a slot are left out, those of weight
// 0 are not (0 times a NaN).
struct Merged {
    float m = -INFINITY, l = 0.f, o[4] = {};
    template <int N>
    __device__ __forceinline__ void add(const float2 (&ml)[N], const float4 (&x)[N]) {
        float mx = m;
#pragma unroll
        for (int i = 0; i < N; ++i) mx = fmaxf(mx, ml[i].x);
        const float mu = mx == -INFINITY ? 0.f : mx, f0 = exp2_fast(m - mu);
        m = mx;
        l *= f0;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ml[i].x == -INFINITY) continue;
            const float f = exp2_fast(ml[i].x - mu);
            l += f * ml[i].y;
            o[0] += f * x[i].x;
            o[1] += f * x[i].y;
            o[2] += f * x[i].z;
            o[3] += f * x[i].w;
        }
    }
    __device__ __forceinline__ uint2 result(bool nan) const {
        if (nan) return make_uint2(0x7FC07FC0u, 0x7FC07FC0u);
        const float f = kUnit / l;
        return make_uint2(pack2(o[0] * f, o[1] * f), pack2(o[2] * f, o[3] * f));
    }
};

template <int D, int NT, Cut CUT>
__global__ void __launch_bounds__(Cfg<D, NT, CUT>::THREADS, Cfg<D, NT, CUT>::CTAS) kv4_decode_kernel(
    const __grid_constant__ Args a) {
    using C = Cfg<D, NT, CUT>;
    constexpr bool WIDE = C::WIDE;
    constexpr int W = C::W, KB = C::KB, GR = C::GR, E = D / 32;
    constexpr int KW = D / 32;   // words of a lane's part of a k row (D / 4 values)
    constexpr int VW = D / 64;   // words of a lane's part of a v row (D / 8 values)
    constexpr int V = C::THREADS >= 256 && NT == 1 ? 2 : 4;  // values of a thread where the warps' parts meet
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    int* pre = reinterpret_cast<int*>(smem + C::OFF_PRE);
    uint8_t* s_free = smem + C::OFF_FREE;
    int* s_nan = reinterpret_cast<int*>(smem + C::OFF_NAN);
    int* flag = reinterpret_cast<int*>(smem + C::OFF_FLAG);
    uint16_t* s_q = reinterpret_cast<uint16_t*>(smem + C::OFF_Q);
    float* s_o = reinterpret_cast<float*>(smem + C::OFF_O);
    float2* s_ml = reinterpret_cast<float2*>(smem + C::OFF_ML);
    Segment* segs = reinterpret_cast<Segment*>(smem + C::OFF_SEG);
    static_assert(sizeof(Segment) == 40, "shared memory");
    const uint32_t new_full = base + C::OFF_BAR;
    if (tid == 0) {
        mbar_init(new_full, W);
        fence_mbar_init();
    }
    griddep_wait();
    griddep_launch_dependents();

    // The CTA's share: from block first.lo of item `first` on, and as far as `stop` in the order of the runs.  (Blocks are
    // counted in int: a cache of 2^31 of them would take 2^31 x 4.5 KB / 16 column groups.)
    const int hc = a.Hkv * a.ncg;  // items of a sequence
    const int cta = static_cast<int>(blockIdx.x);
    auto blocks_of = [&](int b, int& h) {
        h = a.d_hist != nullptr ? a.d_hist[b] : a.hist;
        const bool ok = h >= 0 && h <= a.max_len - a.ntok;
        if (!ok && cta == 0) atomicOr(a.err, kDevErrHistRange);
        return ok ? (h + a.ntok + KB - 1) / KB : 0;
    };
    Segment first;
    int stop = 0, each = 0, more = 0;  // runs: CTA j has each blocks, the first `more` one more
    int n = 0;                         // pieces of an item
    bool alone = false;                // runs of whole items
    auto hist_of = [&](int b, int T) { return T * KB - s_free[b] - a.ntok; };
    if (WIDE && a.batch > 1) {
        if (warp == 0) {
            int h = 0;
            const int T = lane < a.batch ? blocks_of(lane, h) : 0;
            first = piece_of(T, h, hc, static_cast<int>(gridDim.x) / hc, C::ALONE, cta, lane);
            if (lane == 0) segs[0] = first;
        }
        __syncthreads();
        first = segs[0];
        n = first.c0;
        if (n == 0) return;
    } else if (WIDE) {
        const int T = blocks_of(0, first.hist), per = static_cast<int>(gridDim.x) / hc;
        if (T == 0) return;
        n = T <= C::ALONE ? 1 : small_ceil_div(T, max(kMinBlocks, small_ceil_div(T, per)));
        first.b = 0;
        first.T = T;
        first.item = small_div(cta, n);
        if (first.item >= hc) return;
        const int piece = cta - first.item * n, whole = small_div(T, n), rest = T - whole * n;
        first.lo = piece * whole + min(piece, rest);
        first.hi = first.lo + whole + (piece < rest ? 1 : 0);
        first.base = piece;
    } else {
        auto cost_of = [&](int b) {  // with s_free
            int h;
            const int T = blocks_of(b, h);
            s_free[b] = static_cast<uint8_t>(T * KB - h - a.ntok);
            return T > 0 ? T + kItemCost : 0;
        };
        if (a.batch > 32) {
            for (int b = tid; b < a.batch; b += C::THREADS) pre[b + 1] = cost_of(b);
            __syncthreads();
        }
        if (warp == 0) {
            int sum = 0, most = 0;
            uint32_t least = ~0u;
            for (int b0 = 0; b0 < a.batch; b0 += 32) {
                int v = 0;
                if (b0 + lane < a.batch) v = a.batch > 32 ? pre[b0 + lane + 1] : cost_of(lane);
                most = max(most, v);
                if (v > 0) least = min(least, static_cast<uint32_t>(v));
                v = warp_scan(v, lane);
                if (b0 + lane < a.batch) pre[b0 + lane + 1] = sum + v;
                sum += __shfl_sync(0xFFFFFFFFu, v, 31);
            }
            most = __reduce_max_sync(0xFFFFFFFFu, most);
            least = __reduce_min_sync(0xFFFFFFFFu, least);
            if (lane == 0) {
                pre[0] = 0;
                flag[0] = most;
                flag[1] = least == static_cast<uint32_t>(most);
            }
        }
        __syncthreads();
        const int total = pre[a.batch] * hc;
        const int nc = min(static_cast<int>(gridDim.x), (total + kMinBlocks - 1) / kMinBlocks);
        if (cta >= nc) return;
        each = total / nc;
        more = total - each * nc;
        // Whole items, one run's worth or so for each CTA, where the CTA with the most has little more than its run.  Even
        // lengths (32 / 8 heads, us): 64 x 200 tokens 15.4 cut and 10.1 whole, 64 x 1000 27.6 and 23.4, 16 x 200 10.6 and
        // 8.7; but 16 x 500, with an excess of 25, 11.5 and 12.0, and 16 x 1000 13.2 and 18.0.  Mixed lengths
        // add up to more: 64 x 1 .. 300 14.9 and 11.3, 128 x 1 .. 600 26.5 and 25.1, 128 x 1 .. 1000 32.3 and 33.2.
        const int most = flag[0];
        alone = flag[1] ? small_ceil_div(each, most) * most - each <= C::EXCESS : most <= min(each + C::EXCESS, C::LONGEST);
        // The ends of the CTA's run, one in the even lanes and one in the odd; for whole items moved to the nearer end of
        // the item that they are in.
        int r = cta * each + min(cta, more), b = a.batch, item = 0, rem = 0, whole = 1;
        if (lane & 1) r += each + (cta < more ? 1 : 0);
        if (r < total) {
            b = search(pre, a.batch, hc, r);
            whole = pre[b + 1] - pre[b];
            rem = r - pre[b] * hc;
            item = rem / whole;
            rem -= item * whole;
            if (alone) {
                r -= rem;
                if (2 * rem >= whole) {
                    r += whole;
                    if (++item == hc) {
                        item = 0;
                        do ++b;
                        while (b < a.batch && pre[b + 1] == pre[b]);
                        if (b < a.batch) whole = pre[b + 1] - pre[b];
                    }
                }
                rem = 0;
            }
        }
        stop = __shfl_sync(0xFFFFFFFFu, r, 1);
        const int r0 = __shfl_sync(0xFFFFFFFFu, r, 0);
        if (r0 >= stop) return;
        first.b = __shfl_sync(0xFFFFFFFFu, b, 0);
        first.item = __shfl_sync(0xFFFFFFFFu, item, 0);
        first.T = __shfl_sync(0xFFFFFFFFu, whole, 0) - kItemCost;
        first.base = r0 - __shfl_sync(0xFFFFFFFFu, rem, 0) + kItemCost;
        first.lo = max(0, r0 - first.base);
        first.hi = min(first.T, stop - first.base);
        if (first.lo >= first.hi) return;  // the run ends in what the item counts beside its blocks
        first.hist = hist_of(first.b, first.T);
    }
    auto cta_of = [&](int r) {  // whose run has block r
        const int cut = more * (each + 1);
        return r < cut ? r / (each + 1) : more + (r - cut) / each;
    };
    // The item after (b, item), its blocks in the run: false where the run has none of it.
    auto following = [&](int& b, int& item, int& T, int& at, int& hi) {
        at += T + kItemCost;
        if (WIDE || at >= stop) return false;
        if (++item == hc) {
            item = 0;
            do ++b;
            while (pre[b + 1] == pre[b]);
            T = pre[b + 1] - pre[b] - kItemCost;
        }
        hi = min(T, stop - at);
        return true;
    };

    const int G = a.Hq / a.Hkv;
    auto columns = [&](Segment& w) {
        w.head = a.ncg == 1 ? w.item : w.item / a.ncg;
        w.c0 = a.ncg == 1 ? 0 : (w.item - w.head * a.ncg) * 16;
        w.ncol = min(16, G * a.ntok - w.c0);
    };
    auto token = [&](const Segment& w, int col) { return small_div(w.c0 + col, G); };
    auto row_of = [&](const Segment& w, int col) {  // of q and out, in rows of D
        const int i = token(w, col);
        return (static_cast<size_t>(w.b) * a.ntok + i) * a.Hq + w.head * G + (w.c0 + col - i * G);
    };
    // q of an item's columns and its rows of the tables: loaded early, a load waits behind the copies in flight
    constexpr int QN = (C::COLS * (D / 4) + C::THREADS - 1) / C::THREADS;
    uint32_t qx[QN], qy[QN];
    float2 qc[QN], qs[QN];
    auto load_q = [&](const Segment& w) {
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int u = tid + i * C::THREADS, col = u / (D / 4), j = u % (D / 4) * 2;
            qx[i] = qy[i] = 0;  // columns that do not exist
            qc[i] = qs[i] = make_float2(0.f, 0.f);
            if (col < w.ncol) {
                const uint16_t* src = a.q + row_of(w, col) * D + j;
                const size_t p = static_cast<size_t>(w.hist + token(w, col)) * (D / 2) + j;
                qx[i] = __ldg(reinterpret_cast<const uint32_t*>(src));
                qy[i] = __ldg(reinterpret_cast<const uint32_t*>(src + D / 2));
                qc[i] = __ldg(reinterpret_cast<const float2*>(a.cos_tab + p));
                qs[i] = __ldg(reinterpret_cast<const float2*>(a.sin_tab + p));
            }
        }
    };
    auto store_q = [&]() {  // rotated and rounded to bf16
#pragma unroll
        for (int i = 0; i < QN; ++i) {
            const int u = tid + i * C::THREADS, col = u / (D / 4), j = u % (D / 4) * 2;
            if (col >= C::COLS) break;
            const float x0 = __uint_as_float(qx[i] << 16), x1 = __uint_as_float(qx[i] & 0xFFFF0000u);
            const float y0 = __uint_as_float(qy[i] << 16), y1 = __uint_as_float(qy[i] & 0xFFFF0000u);
            *reinterpret_cast<uint32_t*>(s_q + col * C::QS + j) =
                pack2(__fsub_rn(__fmul_rn(x0, qc[i].x), __fmul_rn(y0, qs[i].x)),
                      __fsub_rn(__fmul_rn(x1, qc[i].y), __fmul_rn(y1, qs[i].y)));
            *reinterpret_cast<uint32_t*>(s_q + col * C::QS + j + D / 2) =
                pack2(__fadd_rn(__fmul_rn(y0, qc[i].x), __fmul_rn(x0, qs[i].x)),
                      __fadd_rn(__fmul_rn(y1, qc[i].y), __fmul_rn(x1, qs[i].y)));
        }
    };
    // One warp: an item's q, table rows and new k and v into L2.
    auto prefetch = [&](const Segment& w) {
        constexpr int LINES = D / 64;  // of a row of D bf16 or D / 2 floats
        auto line = [](const void* p, int i) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t*>(p) + 128 * i));
        };
        for (int i = lane; i < w.ncol * LINES; i += 32) line(a.q + row_of(w, i / LINES) * D, i % LINES);
        for (int i = lane; i < a.ntok * 4 * LINES; i += 32) {
            const int tok = i / (4 * LINES), kind = i / LINES % 4;
            const size_t row = (static_cast<size_t>(w.b) * a.ntok + tok) * a.Hkv + w.head, p = static_cast<size_t>(w.hist) + tok;
            if (kind < 2) line((kind == 0 ? a.cos_tab : a.sin_tab) + p * (D / 2), i % LINES);
            else if (w.hi == w.T) line((kind == 2 ? a.k_new : a.v_new) + row * D, i % LINES);
        }
    };
    auto new_from = [&](const Segment& w) { return max(w.hist, w.lo * KB); };  // positions of the new tokens in its blocks
    auto new_to = [&](const Segment& w) { return min(w.hist + a.ntok, w.hi * KB); };
    columns(first);
    load_q(first);
    if (warp == W - 1) prefetch(first);

    // The warp's copies run two blocks ahead of it: block blk_next of an item is next, off_next its byte in
    // the codes (an eighth of it: in the scales).  A group of copies is committed for every block, or an empty one.
    static_assert(C::STAGES == 2 && C::ROW == 8 * 2 * GR, "stages alternate; codes and scales share an offset");
    const uint32_t s_warp = base + static_cast<uint32_t>(warp * C::STAGES * C::STAGE);
    int b_next = first.b, item_next = first.item, T_next = first.T, base_next = first.base, hi_next = first.hi;
    int blk_next = first.lo + warp;
    size_t off_next = 0;
    bool placed = false, ended = false;
    auto issue = [&](uint32_t stage) {
        while (!ended && blk_next >= hi_next) {
            if (!following(b_next, item_next, T_next, base_next, hi_next)) ended = true;
            blk_next = warp;
            placed = false;
        }
        if (!ended) {
            if (!placed) {
                const int head = a.ncg == 1 ? item_next : item_next / a.ncg;
                off_next = ((static_cast<size_t>(b_next) * a.Hkv + head) * a.lp + static_cast<size_t>(blk_next) * KB) * C::ROW +
                           16 * lane;
                placed = true;
            }
            const uint32_t dst = stage + 16 * lane;
            const uint8_t* k = a.c.k_codes + off_next;
            const uint8_t* v = a.c.v_codes + off_next;
#pragma unroll
            for (int i = 0; i < C::CODES; i += 512) {
                copy16(dst + i, k + i);
                copy16(dst + C::CODES + i, v + i);
            }
            // half the lanes the scales of k, half those of v
            const size_t at = ((off_next - 16 * lane) >> 3) + 16 * (lane & 15);
            copy16(dst + 2 * C::CODES, reinterpret_cast<const uint8_t*>(lane < 16 ? a.c.k_scales : a.c.v_scales) + at);
            blk_next += W;
            off_next += static_cast<size_t>(W) * C::CODES;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    issue(s_warp);

    uint32_t st_off = 0;  // of the warp's next block
    uint32_t new_phase = 0;
    // Staged row of new token i, k (0) or v (1): in the O buffer, not yet written, of the warp that has its block.
    auto staged_row = [&](const Segment& w, int i, int kind) {
        const int owner = (((w.hist + i) / KB) - w.lo) % W;
        return smem + C::OFF_O + owner * C::O_BYTES + (2 * i + kind) * C::NEW;
    };
    // The merge of an item's parts by its last CTA: `subs` threads per four values, every subs-th part each.
    auto merge = [&](const Segment& w, int j0, int j1) {
        if (tid == 0) a.counters[static_cast<size_t>(w.b) * hc + w.item] = 0;
        const int vals = w.ncol * (D / 4), subs = max(1, min(C::THREADS / vals, j1 - j0 + 1));
        float4* s_x = reinterpret_cast<float4*>(s_o);
        float2* s_y = reinterpret_cast<float2*>(s_x + C::THREADS);
        for (int u0 = 0; u0 < vals; u0 += C::THREADS) {  // one turn where subs > 1
            const int sub = subs > 1 ? tid / vals : 0, u = u0 + tid - sub * vals;
            const int col = u / (D / 4), d = u % (D / 4) * 4;
            Merged acc;
            int nan = kNone;
            if (sub < subs && u < vals)
#pragma unroll 1
                for (int j = j0 + sub; j <= j1; j += C::BATCH * subs) {
                    float2 ml[C::BATCH];
                    float4 x[C::BATCH];
#pragma unroll
                    for (int i = 0; i < C::BATCH; ++i) {
                        const int from = min(j + i * subs, j1), row = (2 * from + (from == j0 ? 1 : 0)) * 16 + col;
                        ml[i] = __ldcg(reinterpret_cast<const float2*>(a.part_ml) + row);
                        x[i] = __ldcg(reinterpret_cast<const float4*>(a.part_o + static_cast<size_t>(row) * D + d));
                        if (a.ntok > 1) nan = min(nan, __ldcg(a.part_nan + 4 * (row / 16) + d / kKv4Group));
                        if (j + i * subs > j1) ml[i].x = -INFINITY;
                    }
                    acc.add(ml, x);
                }
            if (subs > 1) {
                if (sub > 0 && sub < subs) {
                    s_x[tid] = make_float4(acc.o[0], acc.o[1], acc.o[2], acc.o[3]);
                    s_y[tid] = make_float2(acc.m == INFINITY ? acc.m : mark(acc.m, acc.l), acc.l);
                    if (nan < kNone) atomicMin(&s_nan[d / kKv4Group], nan);
                }
                __syncthreads();
                if (sub == 0)
                    for (int i = 1; i < subs; ++i) {
                        const float2 ml[1] = {s_y[tid + i * vals]};
                        const float4 x[1] = {s_x[tid + i * vals]};
                        acc.add(ml, x);
                    }
                nan = min(nan, s_nan[d / kKv4Group]);
            }
            if (sub == 0 && u < vals && acc.m != INFINITY)
                *reinterpret_cast<uint2*>(a.out + row_of(w, col) * D + d) = acc.result(nan > 0 && nan <= token(w, col));
        }
    };

    if (tid == 0) segs[1].b = -1;
    Segment w = first;
    bool first_turn = true;
    for (bool final_turn = false; !final_turn;) {
        __syncthreads();  // the buffers of the item before are free
        store_q();
        if (tid < 4) s_nan[tid] = kNone;
        if (tid == 0) {
            segs[0] = w;
            flag[2] = 0;
        }
        __syncthreads();
        if (first_turn) issue(s_warp + C::STAGE);
        const Segment& now = segs[0];  // what the walk needs no more is read again after it
        {
            // the new tokens whose slots lie in the segment's blocks, a warp per row of k or v
            const int new0 = new_from(w), new1 = new_to(w);
            if (new0 < new1) {
                for (int u = W - 1 - warp; u < 2 * (new1 - new0); u += W) {
                    const int p = new0 + u / 2, i = p - w.hist;
                    const size_t src = ((static_cast<size_t>(w.b) * a.ntok + i) * a.Hkv + w.head) * D;
                    const size_t slot = (static_cast<size_t>(w.b) * a.Hkv + w.head) * a.lp + p;
                    uint8_t* staged = staged_row(w, i, u & 1);
                    uint32_t x[E / 2];
                    load_row<E / 2>(((u & 1) ? a.v_new : a.k_new) + src, lane, x);
                    if (u & 1) {
                        const bool nan = put_row<D>(x, lane, a.c.v_codes + slot * C::ROW, a.c.v_scales + slot * GR, staged);
                        if (nan && lane % (kKv4Group / E) == 0) atomicMin(&s_nan[lane / (kKv4Group / E)], i);
                    } else {
                        const float turn = lane < 16 ? -1.f : 1.f;  // x c - y s in the first half, x c + y s in the second
#pragma unroll
                        for (int e = 0; e < E / 2; ++e) {
                            const size_t j = static_cast<size_t>(p) * (D / 2) + (lane & 15) * E + 2 * e;
                            const float2 cs = __ldg(reinterpret_cast<const float2*>(a.cos_tab + j));
                            const float2 sn = __ldg(reinterpret_cast<const float2*>(a.sin_tab + j));
                            const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, x[e], 16);
                            x[e] = pack2(__fadd_rn(__fmul_rn(bf_lo(x[e]), cs.x), turn * __fmul_rn(bf_lo(y), sn.x)),
                                         __fadd_rn(__fmul_rn(bf_hi(x[e]), cs.y), turn * __fmul_rn(bf_hi(y), sn.y)));
                        }
                        put_row<D>(x, lane, a.c.k_codes + slot * C::ROW, a.c.k_scales + slot * GR, staged);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(new_full);
            }
            first_turn = false;
            if (warp == 0 && following(w.b, w.item, w.T, w.base, w.hi)) {
                w.hist = hist_of(w.b, w.T);
                columns(w);
                prefetch(w);
            }
        }
        const int hist = now.hist, hi = now.hi;

        // Q^T's B fragments: lane (g, t) holds values D/4 t .. D/4 t + D/4 - 1 of column g (+ 8 n); step s of the
        // products takes values 4 s .. 4 s + 3 of them.  qz: minus their sum in three parts.
        uint32_t qb[NT][2 * KW][2], qz[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t row = base + C::OFF_Q + ((g + 8 * n) * C::QS + (D / 4) * t) * 2;
            float sum_q = 0.f;
#pragma unroll
            for (int s = 0; s < 2 * KW; ++s) {
                lds<2>(row + 8 * s, qb[n][s]);
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    sum_q += __uint_as_float(qb[n][s][e] << 16) + __uint_as_float(qb[n][s][e] & 0xFFFF0000u);
            }
            const float p0 = round_bf16(-sum_q), p1 = round_bf16(-sum_q - p0), p2 = (-sum_q - p0) - p1;
            qz[n][0] = pack2(p0, p1);
            qz[n][1] = pack2(p2, 0.f);
        }
        float o[NT][4 * VW][4] = {}, sum[NT][4] = {};
        // of columns 2 t and 2 t + 1 (+ 8 n): the running maximum m of the scores, m log2 e / sqrt D (0 while m
        // is -inf) less kLift, and the last slot that the column sees
        float m[NT][2], ms[NT][2];
        int lim[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = 8 * n + 2 * t + e;
                m[n][e] = -INFINITY;
                ms[n][e] = -kLift;
                lim[n][e] = hist + min(small_div((a.ncg == 1 ? 0 : now.item % a.ncg * 16) + col, G), a.ntok - 1);
            }

        int blk = now.lo + warp;
        const bool has_blocks = blk < hi;
        for (; blk < hi; blk += W) {
            const int k0 = blk * KB;
            const uint32_t s_k = s_warp + st_off;
            const uint32_t s_v = s_k + C::CODES, s_ks = s_v + C::CODES, s_vs = s_ks + C::SCALES;
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncwarp();
            const bool tail = k0 + KB > hist;  // the block holds slots of new tokens, or none at all
            if (tail) {  // the staged rows into the block
                if (!mbar_wait(new_full, new_phase, nullptr, a.wait_ns)) {
                    record_dev_err(a.err, kDevErrTimeout);
                    flag[2] = 1;
                }
                const int lo = max(k0, hist), hi = min(k0 + KB, hist + a.ntok);
                for (int p = lo; p < hi; ++p)
#pragma unroll
                    for (int kind = 0; kind < 2; ++kind) {
                        const uint32_t* src = reinterpret_cast<const uint32_t*>(staged_row(now, p - hist, kind));
                        uint8_t* dst = smem + (s_k - base);
                        if (lane < C::ROW / 4)
                            reinterpret_cast<uint32_t*>(dst + kind * C::CODES + (p - k0) * C::ROW)[lane] = src[lane];
                        else if (lane < C::NEW / 4)
                            reinterpret_cast<uint32_t*>(dst + 2 * C::CODES + kind * C::SCALES +
                                                        (p - k0) * GR * 2)[lane - C::ROW / 4] = src[lane];
                    }
                __syncwarp();
            }
            const int last = hist + a.ntok - 1 - k0;  // last slot of the block that holds a token
#pragma unroll 1
            for (int half = 0; half < KB / 32; ++half) {
                if (32 * half > last) break;
                // scores of 32 slots: lane (g, t) has slots g, g + 8 of each 16, columns 2 t, 2 t + 1 (+ 8 n)
                float s[2][NT][4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t w[2][KW];
                    Pair p[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int key = 32 * half + 16 * j + 8 * e + g;
                        lds<KW>(s_k + key * C::ROW + t * (KW * 4), w[e]);
                        p[e] = pair_of(__byte_perm(lds16(s_ks + (key * GR + t * GR / 4) * 2), 0, 0x1010));
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_first(s[j][n], p[0].zs, p[1].zs, p[0].zs, p[1].zs, qz[n][0], qz[n][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 2 * KW; ++i) {
                        const uint32_t w0 = w[0][i / 2], w1 = w[1][i / 2];
                        const uint32_t x0 = code2(w0, w0 >> 8, 2 * (i % 2), p[0]), x1 = code2(w1, w1 >> 8, 2 * (i % 2), p[1]),
                                       x2 = code2(w0, w0 >> 8, 2 * (i % 2) + 1, p[0]),
                                       x3 = code2(w1, w1 >> 8, 2 * (i % 2) + 1, p[1]);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma(s[j][n], x0, x1, x2, x3, qb[n][i][0], qb[n][i][1]);
                    }
                }
                bool moves = false;
                float mx[NT][2];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (tail)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    if (k0 + 32 * half + 16 * j + 8 * h + g > lim[n][e]) s[j][n][2 * h + e] = -INFINITY;
                        mx[n][e] = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e]));
                        moves |= mx[n][e] > m[n][e] + a.move;
                    }
                if (__any_sync(0xFFFFFFFFu, moves)) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float x = mx[n][e];
#pragma unroll
                            for (int mask = 4; mask <= 16; mask <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, mask));
                            x = fmaxf(x, m[n][e]);
                            const float f = m[n][e] == x ? 1.f : exp2_fast((m[n][e] - x) * a.scale_log2);
                            m[n][e] = x;
                            ms[n][e] = (x == -INFINITY ? 0.f : x * a.scale_log2) - kLift;
                            sum[n][e] *= f;
#pragma unroll
                            for (int i = 0; i < 4 * VW; ++i) {
                                o[n][i][e] *= f;
                                o[n][i][2 + e] *= f;
                            }
                        }
                }
                uint32_t pb[NT][C::PARTS][4];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float* x = &s[j / 2][n][2 * (j % 2)];
                        const float p0 = exp2_fast(fmaf(x[0], a.scale_log2, -ms[n][0]));
                        const float p1 = exp2_fast(fmaf(x[1], a.scale_log2, -ms[n][1]));
                        const uint32_t hi = pack2(p0, p1);
                        pb[n][0][j] = transpose8(hi);
                        if constexpr (C::PARTS == 2) {
                            pb[n][1][j] = transpose8(pack2(p0 - bf_lo(hi), p1 - bf_hi(hi)));
                            sum[n][0] += p0;
                            sum[n][1] += p1;
                        }
                    }
#pragma unroll
                for (int k = 0; k < 2; ++k) {  // 16 slots
                    const int key = 32 * half + 16 * k + 2 * t;
                    uint32_t w[4][VW], sc[4];  // slots 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = key + (e & 1) + 8 * (e >> 1);
                        lds<VW>(s_v + row * C::ROW + g * (VW * 4), w[e]);
                        sc[e] = lds16(s_vs + (row * GR + g * GR / 8) * 2);
                    }
                    if (tail) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int row = key + (e & 1) + 8 * (e >> 1);
                            if (row > last || (sc[e] >= kTooLarge && k0 + row > hist)) sc[e] = 0;
                        }
                    }
                    Pair p01 = pair_of(__byte_perm(sc[0], sc[1], 0x5410)), p23 = pair_of(__byte_perm(sc[2], sc[3], 0x5410));
                    p01.zs ^= 0x80008000u;
                    p23.zs ^= 0x80008000u;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if constexpr (C::PARTS == 1)
                            mma(sum[n], kOnes, kOnes, kOnes, kOnes, pb[n][0][2 * k], pb[n][0][2 * k + 1]);
#pragma unroll
                    for (int v = 0; v < VW; ++v) {
                        const uint32_t a01 = __byte_perm(w[0][v], w[1][v], 0x5410), b01 = __byte_perm(w[0][v], w[1][v], 0x7632);
                        const uint32_t a23 = __byte_perm(w[2][v], w[3][v], 0x5410), b23 = __byte_perm(w[2][v], w[3][v], 0x7632);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t x0 = value2(a01, a01 >> 8, i, p01), x1 = value2(b01, b01 >> 8, i, p01),
                                           x2 = value2(a23, a23 >> 8, i, p23), x3 = value2(b23, b23 >> 8, i, p23);
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int h = 0; h < C::PARTS; ++h)
                                    mma(o[n][4 * v + i], x0, x1, x2, x3, pb[n][h][2 * k], pb[n][h][2 * k + 1]);
                        }
                    }
                }
            }
            __syncwarp();
            issue(s_k);
            st_off = C::STAGE - st_off;
        }

        if constexpr (C::PARTS == 2) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int mask = 4; mask <= 16; mask <<= 1) sum[n][e] += __shfl_xor_sync(0xFFFFFFFFu, sum[n][e], mask);
        }
        // The warps' parts meet.  Lane (g, t) holds columns 2 t, 2 t + 1 (+ 8 n) of values D/8 g .. D/8 g + D/8 - 1.
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = warp * C::COLS + 8 * n + 2 * t + e;
                if (has_blocks) {
                    float* dst = s_o + col * C::OS + (D / 8) * g;
#pragma unroll
                    for (int i = 0; i < 2 * VW; ++i)
                        *reinterpret_cast<float4*>(dst + 4 * i) =
                            make_float4(o[n][2 * i][e], o[n][2 * i][2 + e], o[n][2 * i + 1][e], o[n][2 * i + 1][2 + e]);
                }
                if (g == 0) s_ml[col] = make_float2(mark(m[n][e] * a.scale_log2, sum[n][e]), sum[n][e]);
            }
        w = now;
        final_turn = !following(w.b, w.item, w.T, w.base, w.hi);
        if (!final_turn) {
            w.lo = 0;
            w.hist = hist_of(w.b, w.T);
            columns(w);
            load_q(w);
        }
        __syncthreads();
        if (new_from(now) < new_to(now)) new_phase ^= 1u;
        const int j0 = WIDE ? cta - now.base : alone ? cta : cta_of(now.base);  // the CTAs that share the item
        const int j1 = WIDE ? j0 + n - 1 : alone ? cta : cta_of(now.base + now.T - 1);
        const int part = 2 * cta + (cta == j0 ? 1 : 0);
        const bool gave_up = flag[2] != 0;
        const int vals = gave_up && j0 == j1 ? 0 : now.ncol * (D / V);
        for (int u = tid; u < vals; u += C::THREADS) {
            const int col = u / (D / V), d = u % (D / V) * V;
            float f[W], mx = -INFINITY, l = 0.f, acc[V] = {};
#pragma unroll
            for (int w = 0; w < W; ++w) {
                f[w] = s_ml[w * C::COLS + col].x;
                mx = fmaxf(mx, f[w]);
            }
            const float mu = mx == -INFINITY ? 0.f : mx;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                if (f[w] == -INFINITY) continue;  // a warp without blocks wrote nothing else
                f[w] = exp2_fast(f[w] - mu);
                l += f[w] * s_ml[w * C::COLS + col].y;
                const float* x = s_o + (w * C::COLS + col) * C::OS + d;
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += f[w] * x[e];
            }
            if (j0 == j1) {
                const int from = s_nan[d / kKv4Group];
                const bool nan = from > 0 && from <= token(now, col);
                const float r = kUnit / l;
#pragma unroll
                for (int e = 0; e < V; e += 2)
                    *reinterpret_cast<uint32_t*>(a.out + row_of(now, col) * D + d + e) =
                        nan ? 0x7FC07FC0u : pack2(acc[e] * r, acc[e + 1] * r);
            } else {
                float* dst = a.part_o + (static_cast<size_t>(part) * 16 + col) * D + d;
#pragma unroll
                for (int e = 0; e < V; e += 2) *reinterpret_cast<float2*>(dst + e) = make_float2(acc[e], acc[e + 1]);
                if (d == 0) reinterpret_cast<float2*>(a.part_ml)[part * 16 + col] = make_float2(gave_up ? INFINITY : mark(mx, l), l);
            }
        }
        if (j0 != j1 && tid < 4) a.part_nan[4 * part + tid] = s_nan[tid];
        if (!final_turn) {
            // a part of an item that began in an earlier CTA is counted at the end: a fence here would hold up the walk
            if (tid == 0 && j0 != j1) segs[1] = now;
            continue;
        }
        __syncthreads();  // the CTA's parts are complete
        const Segment& held = segs[1];
        if (j0 == j1 && held.b < 0) break;
        if (tid == 0) {
            auto last = [&](const Segment& x, int parts) {
                return add_acq_rel(a.counters + static_cast<size_t>(x.b) * hc + x.item, 1) == parts - 1;
            };
            flag[0] = held.b >= 0 && last(held, cta_of(held.base + held.T - 1) - cta_of(held.base) + 1);
            flag[1] = j0 != j1 && last(now, j1 - j0 + 1);
        }
        __syncthreads();
        if (flag[1]) merge(now, j0, j1);
        if (flag[0]) {
            __syncthreads();
            if (tid < 4) s_nan[tid] = kNone;
            __syncthreads();
            merge(held, cta_of(held.base), cta_of(held.base + held.T - 1));
        }
    }
}

template <int D, int NT, Cut CUT>
cudaError_t launch(const Args& a, int num_sms, cudaStream_t st) {
    using C = Cfg<D, NT, CUT>;
    const long long most = static_cast<long long>(a.batch) * a.Hkv * a.ncg * ((a.max_len + C::KB - 1) / C::KB + kItemCost);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min<long long>(num_sms * C::CTAS, most)));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv4_decode_kernel<D, NT, CUT>, a);
}

template <int D, int NT, Cut CUT>
cudaError_t configure() {
    return cudaFuncSetAttribute(kv4_decode_kernel<D, NT, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                Cfg<D, NT, CUT>::BYTES);
}

// Pieces or runs (the lengths are not known here).  Calls in a graph, 4 query heads per kv head, histories of 8000,
// pieces against runs: 8 items 9.1 and 14.8 us, 32 15.0 and 16.7, 64 21.9 and 23.7, 128 32.9 and 36.3; with mixed
// lengths up to 8000, which pieces of whole blocks divide worse the fewer there are per item, 64 16.7 and 17.0,
// 128 28.3 and 24.1.
// With up to one item per SM and more than 8 columns, runs of CTAs of 8 warps, one per SM, instead of 4, two or three
// (head_dim 128, 4 tokens for 16 sequences, 8 kv heads): over 1000 tokens 12.9 and 19.0 us, over 8000 53.3 and 56.1, mixed
// up to 300 9.7 and 11.8, up to 4000 27.4 and 29.8.  (With up to 8 columns such runs of 12 warps take 9.5 us for 12.8
// where 16 sequences have 1000 tokens each, but 14.5 for 11.0 with mixed lengths up to 1000, 28.3 for 24.5 up to 8183.)
template <int D, int NT>
cudaError_t launch_for(const Args& a, int num_sms, cudaStream_t st) {
    const int items = a.batch * a.Hkv * a.ncg;
    if (a.batch <= 32 && 2 * items <= num_sms) return launch<D, NT, kPieces>(a, num_sms, st);
    if constexpr (NT == 2)
        if (items <= num_sms) return launch<D, NT, kRunsFew>(a, num_sms, st);
    return launch<D, NT, kRuns>(a, num_sms, st);
}

}  // namespace

cudaError_t configure_kv4_decode() {
    cudaError_t e = cudaSuccess;
    for (auto fn : {configure<128, 1, kPieces>, configure<128, 1, kRuns>, configure<128, 2, kPieces>, configure<128, 2, kRunsFew>,
                    configure<128, 2, kRuns>, configure<64, 1, kPieces>, configure<64, 1, kRuns>, configure<64, 2, kPieces>,
                    configure<64, 2, kRunsFew>, configure<64, 2, kRuns>})
        if (e == cudaSuccess) e = fn();
    return e;
}

cudaError_t launch_kv4_decode(const Shape& s, const uint16_t* q, const uint16_t* k_new, const uint16_t* v_new,
                              const int32_t* d_hist, int hist, int ntok, const Kv4Cache& c, const float* cos_tab,
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
        a.d_hist = d_hist == nullptr ? nullptr : d_hist + b0;
        a.hist = hist;
        a.lp = kv4_slots(s.max_len);
        const size_t slots = heads * a.lp;
        a.c = Kv4Cache{c.k_codes + slots * (D / 2), c.k_scales + slots * (D / kKv4Group), c.v_codes + slots * (D / 2),
                       c.v_scales + slots * (D / kKv4Group)};
        a.cos_tab = cos_tab;
        a.sin_tab = sin_tab;
        a.part_o = part_o;
        a.part_ml = part_ml;
        a.part_nan = reinterpret_cast<int*>(part_ml + static_cast<size_t>(num_sms) * 4 * 2 * 16 * 2);
        a.counters = counters;
        a.err = err;
        a.wait_ns = wait_ns;
        a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim))) * kUnit;
        a.move = 8.f / a.scale_log2;
        a.batch = std::min(kMaxSeqs, s.batch - b0);
        a.ntok = ntok;
        a.Hq = s.n_q_heads;
        a.Hkv = s.n_kv_heads;
        a.max_len = s.max_len;
        a.ncg = (cols + 15) / 16;
        const cudaError_t e = D == 128 ? (cols <= 8 ? launch_for<128, 1>(a, num_sms, st) : launch_for<128, 2>(a, num_sms, st))
                                       : (cols <= 8 ? launch_for<64, 1>(a, num_sms, st) : launch_for<64, 2>(a, num_sms, st));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace attn
