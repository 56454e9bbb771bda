// tree_decode.cu -- attention of a few new tokens per sequence, a chain or a tree, over the cache and under an optional sliding
// window, with the append of the new tokens and the merge of the splits fused in; and the accepted tokens' move to the end
// of the history.
//
// What a query sees: tree.cuh.  A (sequence, kv head) has n G rows (token, query head of the group), token-major; a row
// group is NT = 1 or 2 tiles of 128 of them.  A tile's rows are the M of the MMAs, a thread's row is its TMEM lane, and 128 slots
// are a key tile: S = Q K^T [128 x 128], O += P V [128 x D], both in TMEM, P in the first columns of its S.  The tiles
// of a sequence are those of its first `sinks` slots and those from its first token's window to its last new slot; what
// lies between is not read.
//
// The work: the key tiles of all (sequence, kv head) in order, cut into equal runs, one per CTA (of each row group), from
// the lengths on the device.  A run's part of an item is a segment; an item in several runs is merged by all the CTAs that
// have a part of it, each a share of its rows and columns, once all parts are written (a cooperative launch: they wait for one
// another, at the end of their runs).
//
// Warps: 4 NT softmax warps (a tile's rows), one TMA producer, one MMA issuer, two guards.
//   producer  K and V tiles through a ring of slots, in the order K0, K1, V0, K2, V1, ..
//   guards    see every tile between the producer and the issuer.  In a tile that holds slots of new tokens they put those in
//             (k rotated), and write them to the cache; in a V tile that some row does not see whole they look for values
//             that are not finite: 0 x NaN would reach the rows that do not see them.  Those become 0 in shared memory, and
//             the rows that see them add them to their O at the end (a rare path, from global memory).
//   issuer    NT = 1: S(j + 1) before P V(j), two S buffers, so that a softmax runs beside the MMAs; Q and O have two buffers
//             each, for the segments in turn.  NT = 2: the tiles' MMAs alternate, each has one S.
//   softmax   rotate the q rows of the next segment into shared memory, scores -> masked by words of 32 slots (in tiles that
//             need it) -> running maximum, moved lazily (by 2^8) -> P as bf16.
// Roundings: rotated q and k to bf16; a weight P to bf16 for its product with v (the operand's type: 2^-8 of it; the
// sum that O is divided by takes it unrounded); the output.  Scores, maxima, sums and O are floats.
// Every wait is bounded; on expiry the CTA records kDevErrTimeout, lets its copies and MMAs finish, releases TMEM and
// still counts its parts in, so that the counters are zero after every launch.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "internal.h"
#include "sm100_ptx.cuh"
#include "tree.cuh"

namespace attn {
namespace {

constexpr int BM = 128;        // rows per tile (TMEM lanes)
constexpr int BN = 128;        // slots per key tile
constexpr int kMaxSeqs = 128;  // sequences of one launch (their tiles are summed in shared memory)
constexpr uint32_t kTmemCols = 512;  // S [0, 256): two of 128; O [256, 256 + 2 D): two
constexpr uint32_t kTmO = 2 * BN;
constexpr int kFlags = 8;
constexpr int kLonger = 4;  // tiles that a piece may be longer than a run
// Registers with three warpgroups (NT = 2): 168 a thread at launch, of which the producer's group leaves 72 to the others.
constexpr int kLaunchRegs = 168;
constexpr uint32_t kRegsLow = 96, kRegsHigh = 200;
static_assert(128 * kRegsLow + 256 * kRegsHigh <= 384 * kLaunchRegs, "register split exceeds the launch total");

template <int D_, int NT_>
struct Cfg {
    static constexpr int D = D_, NT = NT_;
    static constexpr int SOFT = 4 * NT;  // softmax warps; then the producer, the issuer and two guards
    static constexpr int THREADS = (SOFT + 4) * 32;
    static constexpr int DCH = D / 64;        // 128-byte chunks of a row
    static constexpr int CHUNK = 128 * 128;   // bytes of a chunk of 128 rows
    static constexpr int TILE = DCH * CHUNK;  // of a Q, K or V tile
    static constexpr int NS = D == 128 ? 5 : 10;  // ring slots
    static constexpr int ROWS = NT * BM;          // rows of a group
    static constexpr int OFF_Q = 0;               // two Q tiles: of two segments, or of the two row tiles
    static constexpr int OFF_RING = 2 * TILE;
    static constexpr int OFF_PRE = OFF_RING + NS * TILE;     // int [kMaxSeqs]: key tiles up to and with a sequence's
    static constexpr int OFF_HIST = OFF_PRE + kMaxSeqs * 4;  // int [kMaxSeqs]
    static constexpr int OFF_BAR = OFF_HIST + kMaxSeqs * 4;
    enum { B_FULL = 0, B_READY = NS, B_EMPTY = 2 * NS, B_QREADY = 3 * NS, B_QEMPTY = B_QREADY + 2, B_SFULL = B_QEMPTY + 2,
           B_PFULL = B_SFULL + 2, B_OFULL = B_PFULL + 2, B_OEMPTY = B_OFULL + 2, B_PVDONE = B_OEMPTY + 2, B_DRAIN, NBAR };
    static constexpr int OFF_TMEM = OFF_BAR + NBAR * 8;
    static constexpr int OFF_ABORT = OFF_TMEM + 4;
    // int [kFlags]: the segment, from 1, with a value that is not finite in a masked tile; the guards are at most NS / 2 + 1
    // segments ahead of the softmax
    static constexpr int OFF_FLAG = OFF_ABORT + 4;
    static constexpr int OFF_CUT = OFF_FLAG + kFlags * 4;  // int [2]: tiles of a run (0: pieces), of a piece
    static constexpr int BYTES = OFF_CUT + 8;
    static_assert(NS / 2 + 1 < kFlags, "flags");
    static constexpr int ALLOC = BYTES + 1024;  // slack to align the base to 1024 bytes
    static_assert(ALLOC <= 232448, "shared memory budget of one CTA");
};

struct Args {
    const uint16_t* q;
    const uint16_t* k_new;
    const uint16_t* v_new;
    const int32_t* d_hist;
    const int32_t* parents;
    uint16_t* k_cache;
    uint16_t* v_cache;
    const float* cos_tab;
    const float* sin_tab;
    uint16_t* out;
    float* part_o;   // [2 per CTA][D / 4][ROWS][4]
    float* part_ml;  // [2 per CTA][ROWS][2]
    int* counters;   // per item of a launch, zero between launches
    int* err;
    uint64_t wait_ns;
    float scale_log2;
    int b0, batch;  // sequences b0 .. b0 + batch - 1 are this launch's
    int n, Hq, Hkv, G, max_len, window, sinks;
    int groups, runs;  // row groups; runs of each
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Byte offset of the 16-byte unit with columns [col, col + 8) of row `row` in a tile of 128-byte-swizzled 64-column chunks.
__device__ __forceinline__ uint32_t sw128_offset(int row, int col) {
    return static_cast<uint32_t>((col >> 6) * (128 * 128) + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4));
}

// Key tiles of a sequence: tiles 0 .. ns - 1 (of its sinks), then those from ns + skip on; nt in all.
struct Span {
    int ns, skip, nt;
};
__device__ __forceinline__ Span span_of(int hist, const Args& a) {
    const int lo = max(0, hist - a.window + 1), t_lo = lo / BN;  // (the first token's window is the lowest)
    Span s;
    s.ns = min((min(a.sinks, lo) + BN - 1) / BN, t_lo);
    s.skip = t_lo - s.ns;
    s.nt = (hist + a.n + BN - 1) / BN - s.skip;
    return s;
}

// A CTA's part of an item: its tiles lo .. hi - 1 of nt, in part r_mine - r_first of `parts`.
struct Seg {
    int b, h, hist, ns, skip, lo, hi, nt, first;  // first: the item's tile 0 in the order that runs are cut from
    int r_first, parts;                           // the item's first run or piece, and how many have a part of it
    __device__ __forceinline__ int key(int v) const { return (v < ns ? v : v + skip) * BN; }  // first slot of tile v
    __device__ __forceinline__ bool whole() const { return lo == 0 && hi == nt; }
};

// What a CTA takes.  len > 0: the tiles pos .. end - 1 of all items in order, one of the runs of len tiles.  len = 0: the
// piece pos, the only one, of an item that is cut into pieces of at most `target` tiles.
struct Run {
    int pos, end, len, target, id;
    // The CTA's slot for its part of an item: 0 where the item began by the run's start, 1 where it began in it.
    __device__ __forceinline__ int slot(const Seg& s, int r) const { return len == 0 || s.first <= r * len ? 0 : 1; }
};

// The run's next segment, a converged warp; false: none is left.  pre: tiles (pieces) of the items of sequences .. b.
__device__ __forceinline__ bool next_seg(Run& r, const Args& a, const int* pre, const int* hist_s, int lane, Seg& s) {
    if (r.pos >= r.end) return false;
    int before = 0;
#pragma unroll
    for (int i = 0; i < kMaxSeqs / 32; ++i) before += 32 * i + lane < a.batch && pre[32 * i + lane] <= r.pos;
    s.b = __reduce_add_sync(0xFFFFFFFFu, before);
    const int start = s.b > 0 ? pre[s.b - 1] : 0;
    s.hist = hist_s[s.b];
    const Span p = span_of(s.hist, a);
    s.ns = p.ns;
    s.skip = p.skip;
    s.nt = p.nt;
    if (r.len == 0) {
        s.parts = (p.nt + r.target - 1) / r.target;
        s.h = (r.pos - start) / s.parts;
        s.r_first = start + s.h * s.parts;
        const int i = r.pos - s.r_first;
        s.first = 0;
        s.lo = p.nt * i / s.parts;
        s.hi = p.nt * (i + 1) / s.parts;
        r.pos = r.end;
    } else {
        s.h = (r.pos - start) / p.nt;
        s.first = start + s.h * p.nt;
        s.lo = r.pos - s.first;
        s.hi = min(p.nt, r.end - s.first);
        s.r_first = s.first / r.len;
        s.parts = (s.first + p.nt - 1) / r.len - s.r_first + 1;
        r.pos = s.first + s.hi;
    }
    return true;
}

// The kin of a segment's tokens (tree.cuh), a converged warp.  A sequence that is skipped has none: its keys are walked like any
// other's, and nothing is written.
__device__ __forceinline__ void kin_seg(const Seg& s, const Args& a, int lane, uint64_t (&kin)[2], bool report) {
    const int32_t* parents = a.parents == nullptr ? nullptr : a.parents + static_cast<size_t>(a.b0 + s.b) * a.n;
    const int count = tree_kin(parents, a.n, lane, kin);
    const bool range = count > 0 && s.hist + count > a.max_len;
    if (count < 0 || range) {
        kin[0] = kin[1] = 0;
        if (report && lane == 0) atomicOr(a.err, count < 0 ? kDevErrTree : kDevErrHistRange);
    }
}

// Whether some row may not see some slot of the key tile from slot kb on (the same answer in every warp).
__device__ __forceinline__ bool masked(int kb, int hist, const Args& a) {
    return kb + BN > hist || (kb <= hist + a.n - 1 - a.window && kb + BN > a.sinks);
}

// What a row sees: slots [lo, hist) and [0, first), and the new ones whose bit is set.
struct View {
    int lo, hist, first;
    uint64_t kin;
    // bit e: whether it sees slot k0 + e
    __device__ __forceinline__ uint32_t word(int k0) const {
        auto below = [&](int x) {  // bits of the slots < x
            const int c = min(max(x - k0, 0), 32);
            return static_cast<uint32_t>((1ull << c) - 1);
        };
        uint32_t w = (below(hist) & ~below(lo)) | below(first);
        const int d = k0 - hist;
        if (d >= 0) {
            if (d < 64) w |= static_cast<uint32_t>(kin >> d);
        } else if (d > -32) {
            w |= static_cast<uint32_t>(kin << -d);
        }
        return w;
    }
};

__device__ __forceinline__ View view_of(uint64_t kin, int hist, const Args& a) {
    View v;
    const int depth = __popcll(kin) - 1, pos = hist + depth;
    v.hist = hist;
    v.lo = kin == 0 ? hist : min(max(0, pos - a.window + 1), hist);
    v.first = kin == 0 ? 0 : min(a.sinks, hist);
    // without the kin before the window (the d-th lowest bit is at depth d) that are no sinks
    v.kin = kin;
    uint64_t rest = kin;
    for (int d = 0; d <= pos - a.window - hist; ++d, rest &= rest - 1)
        if (hist + d >= a.sinks) v.kin &= ~(rest & (0 - rest));
    return v;
}

// The rotation of 8 pairs (j, j + D / 2): each product and the difference or sum rounded, then to bf16.
__device__ __forceinline__ void rotate8(const uint4& xa, const uint4& xb, const float4 (&c4)[2], const float4 (&s4)[2], uint4& ya,
                                        uint4& yb) {
    const uint32_t wa[4] = {xa.x, xa.y, xa.z, xa.w}, wb[4] = {xb.x, xb.y, xb.z, xb.w};
    const float c[8] = {c4[0].x, c4[0].y, c4[0].z, c4[0].w, c4[1].x, c4[1].y, c4[1].z, c4[1].w};
    const float s[8] = {s4[0].x, s4[0].y, s4[0].z, s4[0].w, s4[1].x, s4[1].y, s4[1].z, s4[1].w};
    uint32_t va[4], vb[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float lo[2], hi[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float x = t ? bf_hi(wa[e]) : bf_lo(wa[e]), y = t ? bf_hi(wb[e]) : bf_lo(wb[e]);
            lo[t] = __fsub_rn(__fmul_rn(x, c[2 * e + t]), __fmul_rn(y, s[2 * e + t]));
            hi[t] = __fadd_rn(__fmul_rn(y, c[2 * e + t]), __fmul_rn(x, s[2 * e + t]));
        }
        va[e] = pack_bf16x2(lo[0], lo[1]);
        vb[e] = pack_bf16x2(hi[0], hi[1]);
    }
    ya = make_uint4(va[0], va[1], va[2], va[3]);
    yb = make_uint4(vb[0], vb[1], vb[2], vb[3]);
}

// Eight pairs of a row with their cosines and sines, loaded ahead of their use.
template <int D>
struct Eight {
    uint4 xa, xb;
    float4 c[2], s[2];
    __device__ __forceinline__ void load(const uint16_t* row, int jb) {
        xa = __ldg(reinterpret_cast<const uint4*>(row + jb));
        xb = __ldg(reinterpret_cast<const uint4*>(row + jb + D / 2));
    }
    __device__ __forceinline__ void angles(int jb, int pos, const Args& a) {
        const float4* cp = reinterpret_cast<const float4*>(a.cos_tab + static_cast<size_t>(pos) * (D / 2) + jb);
        const float4* sp = reinterpret_cast<const float4*>(a.sin_tab + static_cast<size_t>(pos) * (D / 2) + jb);
        c[0] = __ldg(cp);
        c[1] = __ldg(cp + 1);
        s[0] = __ldg(sp);
        s[1] = __ldg(sp + 1);
    }
};

__device__ __forceinline__ uint64_t kin_of(const uint64_t (&kin)[2], int token) {
    const uint64_t k0 = shfl64(kin[0], token & 31), k1 = shfl64(kin[1], token & 31);
    return token < 32 ? k0 : k1;
}

// One warp's 32 rows (from row r0 of the sequence's (token, head) rows on) of q, rotated, into rows `at` .. of a Q tile, and
// the kin of the segment's tokens.  Rows past the last, and of no token, are left: their scores go nowhere.  `empty` waits until the
// tile may be written, after the first loads.
template <int D, typename F>
__device__ __forceinline__ void stage_q(uint8_t* tile, int at, int r0, const Seg& s, uint64_t (&kin)[2], int lane, const Args& a,
                                        F&& empty) {
    constexpr int U = D / 16, BATCH = 4;  // units of a row
    const int rows = min(32, a.n * a.G - r0);
    const int mine = min(max(r0 + lane, 0), a.n * a.G - 1) / a.G;
    int depth = 0;
    for (int i0 = 0; i0 == 0 || i0 * (32 / U) < rows; i0 += BATCH) {
        Eight<D> x[BATCH];
        int row[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int u = (i0 + i) * 32 + lane;
            row[i] = u / U;
            const int token = __shfl_sync(0xFFFFFFFFu, mine, row[i] & 31);
            if (row[i] >= rows)
                row[i] = -1;
            else
                x[i].load(a.q + ((static_cast<size_t>(a.b0 + s.b) * a.n + token) * a.Hq + s.h * a.G + (r0 + row[i] - token * a.G)) * D,
                          u % U * 8);
        }
        if (i0 == 0) {
            kin_seg(s, a, lane, kin, false);
            const uint64_t k = kin_of(kin, mine);
            depth = k == 0 ? -1 : __popcll(k) - 1;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int d = __shfl_sync(0xFFFFFFFFu, depth, max(row[i], 0) & 31);
            if (d < 0) row[i] = -1;
            if (row[i] >= 0) x[i].angles(((i0 + i) * 32 + lane) % U * 8, s.hist + d, a);
        }
        if (i0 == 0 && !empty()) return;
#pragma unroll
        for (int i = 0; i < BATCH; ++i)
            if (row[i] >= 0) {
                const int jb = ((i0 + i) * 32 + lane) % U * 8;
                rotate8(x[i].xa, x[i].xb, x[i].c, x[i].s, *reinterpret_cast<uint4*>(tile + sw128_offset(at + row[i], jb)),
                        *reinterpret_cast<uint4*>(tile + sw128_offset(at + row[i], jb + D / 2)));
            }
    }
}

// Add to o (columns c0 .. c0 + 31 of a row's O) the values that are not finite of the slots that the row sees in the masked tiles.
template <int D>
__device__ __noinline__ void add_not_finite(float* o, int c0, const View& view, const Seg& s, const Args& a) {
    const size_t head = (static_cast<size_t>(a.b0 + s.b) * a.Hkv + s.h) * a.max_len;
    for (int v = s.lo; v < s.hi; ++v) {
        const int kb = s.key(v);
        if (!masked(kb, s.hist, a)) continue;
        for (int c = 0; c < BN / 32; ++c)
            for (uint32_t w = view.word(kb + 32 * c); w != 0; w &= w - 1) {
                const int slot = kb + 32 * c + __ffs(w) - 1;
                const uint16_t* row = slot < s.hist ? a.v_cache + (head + slot) * D
                                                    : a.v_new + ((static_cast<size_t>(a.b0 + s.b) * a.n + slot - s.hist) * a.Hkv + s.h) * D;
                for (int e = 0; e < 32; ++e) {
                    const float x = __uint_as_float(static_cast<uint32_t>(row[c0 + e]) << 16);
                    if (!isfinite(x)) o[e] += x;
                }
            }
    }
}

__device__ __forceinline__ int load_acquire(const int* p) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

template <int D, int NT>
__global__ void __launch_bounds__(Cfg<D, NT>::THREADS, 1)
    tree_decode_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const Args a) {
    using C = Cfg<D, NT>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* gbase = smem_raw + (base - raw);
    int* pre = reinterpret_cast<int*>(gbase + C::OFF_PRE);
    int* hist_s = reinterpret_cast<int*>(gbase + C::OFF_HIST);
    int* cut = reinterpret_cast<int*>(gbase + C::OFF_CUT);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(gbase + C::OFF_ABORT);
    volatile int* odd_flag = reinterpret_cast<volatile int*>(gbase + C::OFF_FLAG);
    auto bar = [&](int i) -> uint32_t { return base + C::OFF_BAR + 8u * static_cast<uint32_t>(i); };

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kWarpTma = C::SOFT, kWarpMma = C::SOFT + 1, kWarpGuard = C::SOFT + 2;
    const int group = static_cast<int>(blockIdx.x) % a.groups, run_id = static_cast<int>(blockIdx.x) / a.groups;
    const int group_rows = min(C::ROWS, a.n * a.G - group * C::ROWS);
    const int live = NT == 1 || group_rows <= BM ? 1 : 2;  // tiles with rows

    if (warp == kWarpTma && lane == 0) {
        *abort_flag = 0;
        for (int i = 0; i < kFlags; ++i) odd_flag[i] = 0;
        for (int i = 0; i < C::NS; ++i) {
            mbar_init(bar(C::B_FULL + i), 1);
            mbar_init(bar(C::B_READY + i), 2);  // the guards
            mbar_init(bar(C::B_EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::B_QREADY + i), 4 * live);
            mbar_init(bar(C::B_QEMPTY + i), 1);
            mbar_init(bar(C::B_SFULL + i), 1);
            mbar_init(bar(C::B_PFULL + i), 4);
            mbar_init(bar(C::B_OFULL + i), 1);
            mbar_init(bar(C::B_OEMPTY + i), 4);
        }
        mbar_init(bar(C::B_PVDONE), 1);
        mbar_init(bar(C::B_DRAIN), 1);
        fence_mbar_init();
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    // parents on their way while the lengths are
    if (a.parents != nullptr && warp >= kWarpGuard)
        for (int i = (warp - kWarpGuard) * 32 + lane; i * 32 < a.batch * a.n; i += 64)
            asm volatile("prefetch.global.L1 [%0];" ::"l"(a.parents + static_cast<size_t>(a.b0) * a.n + 32 * i));
    if (warp == kWarpMma) {
        tmem_alloc(base + C::OFF_TMEM, kTmemCols);
        tmem_relinquish();
    }
    if (warp == 0) {  // the tiles of the sequences, summed: lane l has sequences 4 l .. 4 l + 3
        constexpr int PER = kMaxSeqs / 32;
        int h[PER], t[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) h[i] = PER * lane + i < a.batch ? __ldg(a.d_hist + a.b0 + PER * lane + i) : 0;
        bool bad = false;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const bool here = PER * lane + i < a.batch, good = h[i] >= 0 && h[i] <= a.max_len;
            bad |= !good;
            t[i] = here && good ? span_of(h[i], a).nt : 0;
            sum += t[i] * a.Hkv;
            hist_s[PER * lane + i] = h[i];
        }
        const int total = __reduce_add_sync(0xFFFFFFFFu, sum);
        // Pieces, if there are CTAs for all and they are hardly longer than the runs would be: a CTA then has but one segment.
        const int len = max((total + a.runs - 1) / a.runs, 1);
        int target = len;
        for (; target <= len + kLonger; target += max(target >> 5, 1)) {
            int pieces = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) pieces += (t[i] + target - 1) / target * a.Hkv;
            if (__reduce_add_sync(0xFFFFFFFFu, pieces) <= a.runs) break;
        }
        const bool in_pieces = target <= len + kLonger;
        sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            sum += (in_pieces ? (t[i] + target - 1) / target : t[i]) * a.Hkv;
            t[i] = sum;
        }
        int upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int u = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += u;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) pre[PER * lane + i] = upto - sum + t[i];
        if (lane == 0) {
            cut[0] = in_pieces ? 0 : len;
            cut[1] = target;
        }
        if (bad && blockIdx.x == 0) atomicOr(a.err, kDevErrHistRange);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<const uint32_t*>(gbase + C::OFF_TMEM);

    Run run;
    run.id = run_id;
    run.len = cut[0];
    run.target = cut[1];
    run.pos = min(run_id * max(run.len, 1), pre[kMaxSeqs - 1]);
    run.end = min(run.pos + max(run.len, 1), pre[kMaxSeqs - 1]);
    const Run run0 = run;
    Seg s;
    uint64_t kin[2];
    // The ring's order of a segment of n tiles: K0, K1, V0, K2, V1, .., V(n - 1); where K(j) and V(j) are in it.
    auto k_at = [](int j) { return j == 0 ? 0 : 2 * j - 1; };
    auto v_at = [](int j, int n) { return min(2 * j + 2, 2 * n - 1); };
    // and what is at place i: tile j, V or not
    auto tile_at = [](int i, int n, bool& is_v) {
        is_v = i == 2 * n - 1 || (i > 0 && i % 2 == 0);
        return i == 2 * n - 1 ? n - 1 : is_v ? i / 2 - 1 : (i + 1) / 2;
    };
    bool ok = true;

    if (warp >= C::SOFT) {
        if constexpr (NT == 2) warpgroup_reg_dec<kRegsLow>();
        if (warp == kWarpTma) {
            // ------------------------------------------------------------ producer
            uint32_t seq = 0;
            while (ok && next_seg(run, a, pre, hist_s, lane, s)) {
                if (lane == 0) {
                    const int n = s.hi - s.lo, head = (a.b0 + s.b) * a.Hkv + s.h;
                    for (int i = 0; i < 2 * n; ++i, ++seq) {
                        const uint32_t st = seq % C::NS;
                        if (seq >= C::NS && !mbar_wait(bar(C::B_EMPTY + st), (seq / C::NS - 1u) & 1u, abort_flag, a.wait_ns)) {
                            ok = false;
                            break;
                        }
                        bool is_v;
                        const int kb = s.key(s.lo + tile_at(i, n, is_v));
                        mbar_arrive_expect_tx(bar(C::B_FULL + st), C::TILE);
#pragma unroll
                        for (int c = 0; c < C::DCH; ++c)
                            tma_load_3d(base + C::OFF_RING + st * C::TILE + c * C::CHUNK, is_v ? &map_v : &map_k, c * 64, kb, head,
                                        bar(C::B_FULL + st));
                    }
                    if (!ok) {
                        *abort_flag = 1;
                        atomicOr(a.err, kDevErrTimeout);
                    }
                }
                ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
            }
            if (lane == 0)  // every copy issued must land before the CTA may exit
                for (uint32_t i = seq >= C::NS ? seq - C::NS : 0; i < seq; ++i)
                    mbar_wait(bar(C::B_FULL + i % C::NS), (i / C::NS) & 1u, nullptr);
        } else if (warp == kWarpMma) {
            // ------------------------------------------------------------ issuer
            constexpr uint32_t kIdS = idesc_bf16_f32(BM, BN, false, false);
            constexpr uint32_t kIdPV = idesc_bf16_f32(BM, D, false, true);
            constexpr uint32_t kHi = desc_hi_sw128(1024);
            const uint32_t q_lo0 = desc_lo_sw128(base + C::OFF_Q, 16);
            const uint32_t k_lo0 = desc_lo_sw128(base + C::OFF_RING, 16);
            const uint32_t v_lo0 = desc_lo_sw128(base + C::OFF_RING, C::CHUNK);
            uint32_t seq = 0, tiles = 0, segs = 0;
            auto issue_s = [&](uint32_t buf, uint32_t q, uint32_t slot) {
                const uint32_t a_lo = q_lo0 + q * (C::TILE >> 4), b_lo = k_lo0 + slot * (C::TILE >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t c = ((kk >> 2) * C::CHUNK + (kk & 3) * 32) >> 4;
                    umma_ss_w(tmem + buf * BN, a_lo + c, kHi, b_lo + c, kHi, kIdS, kk > 0 ? 1u : 0u);
                }
                umma_commit(bar(C::B_SFULL + buf));
            };
            auto issue_pv = [&](uint32_t buf, uint32_t o, bool first, uint32_t slot) {
                const uint32_t b_lo = v_lo0 + slot * (C::TILE >> 4);
#pragma unroll
                for (int kk = 0; kk < BN / 16; ++kk)
                    umma_ts_w(tmem + kTmO + o * D, tmem + buf * BN + kk * 8, b_lo + kk * ((16 * 128) >> 4), kHi, kIdPV,
                              (!first || kk > 0) ? 1u : 0u);
            };
            auto ready = [&](uint32_t at) {
                return mbar_wait(bar(C::B_READY + at % C::NS), (at / C::NS) & 1u, abort_flag, a.wait_ns);
            };
            while (ok && next_seg(run, a, pre, hist_s, lane, s)) {
                if (lane == 0) {
                    const int n = s.hi - s.lo;
                    const uint32_t qb = NT == 1 ? segs & 1u : 0u;
                    ok = mbar_wait(bar(C::B_QREADY + qb), (NT == 1 ? segs >> 1 : segs) & 1u, abort_flag, a.wait_ns);
                    for (int j = 0; j <= n && ok; ++j) {
                        if constexpr (NT == 1) {
                            if (j < n) {
                                const uint32_t at = seq + k_at(j);
                                if (!(ok = ready(at))) break;
                                tc_fence_after();
                                issue_s((tiles + j) & 1u, qb, at % C::NS);
                                umma_commit(bar(C::B_EMPTY + at % C::NS));
                                if (j == n - 1) umma_commit(bar(C::B_QEMPTY + qb));
                            }
                            if (j > 0) {
                                const uint32_t t = tiles + j - 1, at = seq + v_at(j - 1, n);
                                ok = mbar_wait(bar(C::B_PFULL + (t & 1u)), (t >> 1) & 1u, abort_flag, a.wait_ns) && ready(at) &&
                                     (j > 1 || segs < 2 ||
                                      mbar_wait(bar(C::B_OEMPTY + qb), ((segs >> 1) - 1u) & 1u, abort_flag, a.wait_ns));
                                if (!ok) break;
                                tc_fence_after();
                                issue_pv(t & 1u, qb, j == 1, at % C::NS);
                                umma_commit(bar(C::B_PVDONE));
                                umma_commit(bar(C::B_EMPTY + at % C::NS));
                            }
                        } else {
                            const uint32_t ka = seq + k_at(j), va = seq + v_at(j - 1, n);
                            ok = (j == n || ready(ka)) && (j == 0 || ready(va));
                            if (!ok) break;
                            tc_fence_after();
                            for (int t = 0; t < live; ++t) {
                                if (j > 0) {
                                    ok = mbar_wait(bar(C::B_PFULL + t), (tiles + j - 1) & 1u, abort_flag, a.wait_ns) &&
                                         (j > 1 || segs == 0 || mbar_wait(bar(C::B_OEMPTY + t), (segs - 1u) & 1u, abort_flag, a.wait_ns));
                                    if (!ok) break;
                                    tc_fence_after();
                                    issue_pv(t, t, j == 1, va % C::NS);
                                }
                                if (j < n) issue_s(t, t, ka % C::NS);
                            }
                            if (!ok) break;
                            if (j < n) umma_commit(bar(C::B_EMPTY + ka % C::NS));
                            if (j > 0) umma_commit(bar(C::B_EMPTY + va % C::NS));
                            if (j == n - 1) umma_commit(bar(C::B_QEMPTY));
                        }
                    }
                    if (ok) {
                        if constexpr (NT == 1)
                            umma_commit(bar(C::B_OFULL + qb));
                        else
                            for (int t = 0; t < live; ++t) umma_commit(bar(C::B_OFULL + t));
                    } else {
                        *abort_flag = 1;
                        atomicOr(a.err, kDevErrTimeout);
                    }
                    tiles += n;
                    seq += 2 * n;
                    ++segs;
                }
                ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
            }
            if (lane == 0) {  // all tensor-core work must finish before TMEM is released
                umma_commit(bar(C::B_DRAIN));
                mbar_wait(bar(C::B_DRAIN), 0, nullptr);
            }
        } else {
            // ------------------------------------------------------------ guards
            // A guard has the rows of a tile whose bit 2 is its number: the 16-byte units u with u % 64 in its half.
            const int gw = warp - kWarpGuard, me = gw * 32 + lane;
            auto rows_below = [&](int row) { return row / 8 * 4 + min(max(row % 8 - 4 * gw, 0), 4); };  // of this guard's
            uint32_t seq = 0, segs = 0;
            while (ok && next_seg(run, a, pre, hist_s, lane, s)) {
                kin_seg(s, a, lane, kin, group == 0 && warp == kWarpGuard);
                const int n = s.hi - s.lo;
                const size_t head = (static_cast<size_t>(a.b0 + s.b) * a.Hkv + s.h) * a.max_len + s.hist;  // slot of token 0
                for (int i = 0; i < 2 * n && ok; ++i, ++seq) {
                    const uint32_t st = seq % C::NS;
                    bool is_v;
                    const int kb = s.key(s.lo + tile_at(i, n, is_v));
                    uint8_t* tile = gbase + C::OFF_RING + st * C::TILE;
                    const bool mixed = masked(kb, s.hist, a);
                    const int t0 = max(kb - s.hist, 0), t1 = min(kb + BN - s.hist, a.n);  // new tokens of this tile
                    bool there = false;  // the tile has landed
                    auto landed = [&]() {
                        if (!there) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(C::B_FULL + st), (seq / C::NS) & 1u, abort_flag, a.wait_ns));
                        there = true;
                    };
                    if (t1 > t0) {
                        constexpr int U = D / 16, BATCH = 2;
                        const int at0 = s.hist - kb, i0 = rows_below(at0 + t0), units = (rows_below(at0 + t1) - i0) * U;
                        for (int u0 = 0; u0 < units && ok; u0 += 32 * BATCH) {
                            Eight<D> x[BATCH];
                            int token[BATCH];
#pragma unroll
                            for (int e = 0; e < BATCH; ++e) {
                                const int u = u0 + 32 * e + lane, i_row = i0 + u / U;
                                const int t = min(max(i_row / 4 * 8 + 4 * gw + i_row % 4 - at0, 0), a.n - 1);
                                const uint64_t k = kin_of(kin, t);
                                token[e] = u < units && k != 0 ? t : -1;
                                if (token[e] < 0) continue;
                                const size_t row = ((static_cast<size_t>(a.b0 + s.b) * a.n + t) * a.Hkv + s.h) * D;
                                if (is_v) {  // units of k are pairs of 8, of v two times 8 as well
                                    x[e].xa = __ldg(reinterpret_cast<const uint4*>(a.v_new + row + u % U * 8));
                                    x[e].xb = __ldg(reinterpret_cast<const uint4*>(a.v_new + row + u % U * 8 + D / 2));
                                } else {
                                    x[e].load(a.k_new + row, u % U * 8);
                                    x[e].angles(u % U * 8, s.hist + __popcll(k) - 1, a);
                                }
                            }
                            landed();
                            if (!ok) break;
#pragma unroll
                            for (int e = 0; e < BATCH; ++e) {
                                if (token[e] < 0) continue;
                                const int jb = (u0 + 32 * e + lane) % U * 8, row = at0 + token[e];
                                uint4 ya = x[e].xa, yb = x[e].xb;
                                if (!is_v) rotate8(x[e].xa, x[e].xb, x[e].c, x[e].s, ya, yb);
                                *reinterpret_cast<uint4*>(tile + sw128_offset(row, jb)) = ya;
                                *reinterpret_cast<uint4*>(tile + sw128_offset(row, jb + D / 2)) = yb;
                                if (group == 0) {
                                    uint16_t* to = (is_v ? a.v_cache : a.k_cache) + (head + token[e]) * D + jb;
                                    *reinterpret_cast<uint4*>(to) = ya;
                                    *reinterpret_cast<uint4*>(to + D / 2) = yb;
                                }
                            }
                        }
                    }
                    if (ok) landed();
                    if (!ok) break;
                    if (is_v && mixed) {
                        __syncwarp();  // (the rows of new tokens are written)
                        // the products with 0 add up to 0, or to NaN
                        uint4* units = reinterpret_cast<uint4*>(tile);
                        uint32_t sum[4] = {0u, 0u, 0u, 0u};
#pragma unroll 8
                        for (int u = me; u < C::TILE / 16; u += 64) {
                            const uint4 w = units[u];
                            const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum[e]) : "r"(v[e]), "r"(0u));
                        }
                        if (__any_sync(0xFFFFFFFFu, ((sum[0] | sum[1] | sum[2] | sum[3]) & 0x7FFF7FFFu) != 0)) {
                            for (int u = me; u < C::TILE / 16; u += 64) {
                                uint4 w = units[u];
                                uint32_t* v = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if ((v[e] & 0x7F80u) == 0x7F80u) v[e] &= 0xFFFF0000u;
                                    if ((v[e] & 0x7F800000u) == 0x7F800000u) v[e] &= 0x0000FFFFu;
                                }
                                units[u] = w;
                            }
                            odd_flag[segs % kFlags] = static_cast<int>(segs) + 1;
                        }
                    }
                    if (mixed) fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::B_READY + st));
                }
                ++segs;
            }
            if (!ok && lane == 0) {
                *abort_flag = 1;
                atomicOr(a.err, kDevErrTimeout);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax
        if constexpr (NT == 2) warpgroup_reg_inc<kRegsHigh>();
        const int t = warp >> 2;  // row tile
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const int r0 = group * C::ROWS + warp * 32;  // the warp's first row
        const bool rows_on = r0 < a.n * a.G;
        const bool row_on = r0 + lane < a.n * a.G;
        const int token = min(r0 + lane, a.n * a.G - 1) / a.G;
        int did[2] = {0, 0};  // what this warp has counted of the parts at the run's ends
        if (t < live) {
            uint32_t tiles = 0, segs = 0;
            Seg nx;
            uint64_t nkin[2];
            Run ahead = run;
            auto stage = [&](uint32_t seg) {  // q and kin of segment nx
                const uint32_t qb = NT == 1 ? seg & 1u : 0u, use = NT == 1 ? seg >> 1 : seg;
                stage_q<D>(gbase + C::OFF_Q + (NT == 1 ? qb : static_cast<uint32_t>(t)) * C::TILE, (warp & 3) * 32, r0, nx, nkin, lane, a,
                           [&]() {
                               if (use > 0)
                                   ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(C::B_QEMPTY + qb), (use - 1u) & 1u, abort_flag, a.wait_ns));
                               return ok;
                           });
                if (!ok) return;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::B_QREADY + qb));
            };
            bool more = next_seg(ahead, a, pre, hist_s, lane, nx);
            if (more) stage(0);
            while (more && ok) {
                s = nx;
                const uint64_t k = kin_of(nkin, token);
                const bool write = row_on && k != 0;
                const View view = view_of(row_on ? k : 0, s.hist, a);
                float m_run = -INFINITY, l_run = 0.f;  // the reference of P (log2 domain), the sum
                const uint32_t ob = NT == 1 ? segs & 1u : static_cast<uint32_t>(t);
                const uint32_t o_col = tmem + lane_base + kTmO + ob * D;
                for (int v = s.lo; v < s.hi; ++v, ++tiles) {
                    const uint32_t sb = NT == 1 ? tiles & 1u : static_cast<uint32_t>(t);
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(C::B_SFULL + sb), (NT == 1 ? tiles >> 1 : tiles) & 1u, abort_flag, a.wait_ns));
                    if (!ok) break;
                    if (rows_on) {
                        tc_fence_after();
                        const uint32_t s_col = tmem + lane_base + sb * BN;
                        uint32_t r[BN / 32][32];
#pragma unroll
                        for (int c = 0; c < BN / 32; ++c) tmem_ld32(s_col + 32 * c, r[c]);
                        tmem_wait_ld();
                        const int kb = s.key(v);
                        if (masked(kb, s.hist, a)) {
#pragma unroll
                            for (int c = 0; c < BN / 32; ++c) {
                                const uint32_t w = view.word(kb + 32 * c);
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!(w >> e & 1u)) r[c][e] = __float_as_uint(-INFINITY);
                            }
                        }
                        float mxc[BN / 32];  // row maximum: four chains
#pragma unroll
                        for (int c = 0; c < BN / 32; ++c) {
                            mxc[c] = __uint_as_float(r[c][0]);
#pragma unroll
                            for (int e = 1; e < 31; e += 2)
                                mxc[c] = fmax3(mxc[c], __uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1]));
                            mxc[c] = fmaxf(mxc[c], __uint_as_float(r[c][31]));
                        }
                        const float mx = fmaxf(fmaxf(mxc[0], mxc[1]), fmaxf(mxc[2], mxc[3]));
                        const float m_cand = fmaxf(m_run, mx * a.scale_log2);
                        const bool move = m_cand > m_run + 8.f;  // (always with a row's first slot)
                        const float m_new = move ? m_cand : m_run;
                        const float alpha = move ? fast_exp2(m_run - m_new) : 1.f;
                        const float m_ref = m_new == -INFINITY ? 0.f : m_new;  // (no slot seen so far: P = 0)
                        const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), nm2 = make_float2(-m_ref, -m_ref);
                        float2 sum2[BN / 32];
#pragma unroll
                        for (int c = 0; c < BN / 32; ++c) {
                            uint32_t pw[16];
                            float2 acc2 = make_float2(0.f, 0.f);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 x =
                                    ffma2(make_float2(__uint_as_float(r[c][2 * i]), __uint_as_float(r[c][2 * i + 1])), sc2, nm2);
                                const float2 pp = make_float2(fast_exp2(x.x), fast_exp2(x.y));
                                acc2 = ffma2(pp, make_float2(1.f, 1.f), acc2);
                                pw[i] = pack_bf16x2(pp.x, pp.y);
                            }
                            sum2[c] = acc2;
                            tmem_st16(s_col + 16 * c, pw);
                        }
                        const float2 sum2a = make_float2(sum2[0].x + sum2[1].x, sum2[0].y + sum2[1].y);
                        const float2 sum2b = make_float2(sum2[2].x + sum2[3].x, sum2[2].y + sum2[3].y);
                        l_run = l_run * alpha + ((sum2a.x + sum2b.x) + (sum2a.y + sum2b.y));
                        m_run = m_new;
                        // O is rescaled between two P V: with NT = 2 the last one ended before these scores
                        if (NT == 1 && tiles > 0) {
                            ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(C::B_PVDONE), (tiles - 1u) & 1u, abort_flag, a.wait_ns));
                            if (!ok) break;
                            tc_fence_after();
                        }
                        if (v > s.lo && __any_sync(0xFFFFFFFFu, move)) {
#pragma unroll
                            for (int c = 0; c < D / 32; ++c) {
                                uint32_t o[32];
                                tmem_ld32(o_col + 32 * c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                                tmem_st32(o_col + 32 * c, o);
                            }
                        }
                        tmem_wait_st();
                        tc_fence_before();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::B_PFULL + sb));
                }
                if (!ok) break;
                // the next segment's q beside this one's last MMAs
                more = next_seg(ahead, a, pre, hist_s, lane, nx);
                if (more) stage(segs + 1);
                if (!ok) break;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar(C::B_OFULL + ob), (NT == 1 ? segs >> 1 : segs) & 1u, abort_flag, a.wait_ns));
                if (!ok) break;
                const bool whole = s.whole();
                const int slot = run0.slot(s, run_id);
                if (rows_on) {
                    tc_fence_after();
                    const bool odd = odd_flag[segs % kFlags] == static_cast<int>(segs) + 1;
                    const float inv = 1.f / l_run;
                    const int head = s.h * a.G + (r0 + lane - token * a.G);
                    uint16_t* orow = a.out + ((static_cast<size_t>(a.b0 + s.b) * a.n + token) * a.Hq + head) * D;
                    float* part = a.part_o + ((static_cast<size_t>(blockIdx.x) * 2 + slot) * (D / 4) * C::ROWS + warp * 32 + lane) * 4;
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o_col + 32 * c, o);
                        tmem_wait_ld();
                        float f[32];
#pragma unroll
                        for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(o[e]);
                        if (write && odd) {
                            float g[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) g[e] = f[e];
                            add_not_finite<D>(g, 32 * c, view, s, a);
#pragma unroll
                            for (int e = 0; e < 32; ++e) f[e] = g[e];
                        }
                        if (write && whole) {
#pragma unroll
                            for (int e = 0; e < 32; e += 8)
                                *reinterpret_cast<uint4*>(orow + 32 * c + e) =
                                    make_uint4(pack_bf16x2(f[e] * inv, f[e + 1] * inv), pack_bf16x2(f[e + 2] * inv, f[e + 3] * inv),
                                               pack_bf16x2(f[e + 4] * inv, f[e + 5] * inv), pack_bf16x2(f[e + 6] * inv, f[e + 7] * inv));
                        } else if (write) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4)
                                *reinterpret_cast<float4*>(part + static_cast<size_t>(8 * c + e / 4) * C::ROWS * 4) =
                                    make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                        }
                        __syncwarp();
                    }
                    if (write && !whole)
                        *reinterpret_cast<float2*>(a.part_ml + ((static_cast<size_t>(blockIdx.x) * 2 + slot) * C::ROWS + warp * 32 + lane) * 2) =
                            make_float2(m_run, l_run);
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(bar(C::B_OEMPTY + ob));
                    if (!whole) {
                        __threadfence();
                        atomicAdd(a.counters + (s.b * a.Hkv + s.h) * a.groups + group, 1);
                    }
                }
                if (!whole) did[slot] = 1;
                ++segs;
            }
            if (!ok && lane == 0) {
                *abort_flag = 1;
                atomicOr(a.err, kDevErrTimeout);
            }
            // ---- the merges: of the item that began by the run's start, and of the one that goes on past its end
            Run again = run0;
            while (next_seg(again, a, pre, hist_s, lane, s)) {
                if (s.whole()) continue;
                const int slot = run0.slot(s, run_id), r_first = s.r_first, parts = s.parts;
                int* counter = a.counters + (s.b * a.Hkv + s.h) * a.groups + group;
                const int warps = 4 * live, all = parts * warps;
                if (ok && did[slot] == 1) {
                    // (every CTA of the cooperative launch is resident, and none waits before its parts are counted)
                    bool done = load_acquire(counter) >= all;
                    if (!done) {
                        const uint64_t t_0 = globaltimer_ns();
                        do {
                            __nanosleep(32);
                            done = load_acquire(counter) >= all;
                        } while (!done && globaltimer_ns() - t_0 <= a.wait_ns);
                    }
                    ok = __all_sync(0xFFFFFFFFu, done);
                    if (!ok && lane == 0) atomicOr(a.err, kDevErrTimeout);
                }
                if (ok && did[slot] == 1) {
                    const int blocks = (group_rows + 31) / 32, share = (run_id - r_first) * warps + warp;
                    const int blk = share % blocks, part = share / blocks, of = (all - blk + blocks - 1) / blocks;
                    const int row = blk * 32 + lane, R = group * C::ROWS + row;
                    const int tok = min(R, a.n * a.G - 1) / a.G;
                    kin_seg(s, a, lane, kin, false);
                    const uint64_t k = kin_of(kin, tok);  // (by all lanes)
                    const bool write = row < group_rows && k != 0;
                    auto slot_of = [&](int p) {  // of part p
                        const int r = r_first + p;
                        return static_cast<size_t>(r * a.groups + group) * 2 + run0.slot(s, r);
                    };
                    if (write) {
                        // a batch of parts is loaded at once: one after the other, each would wait for its loads
                        constexpr int BATCH = 8;
                        auto load_ml = [&](int p0, float2 (&ml)[BATCH]) {
#pragma unroll
                            for (int i = 0; i < BATCH; ++i)
                                ml[i] = p0 + i < parts ? __ldcg(reinterpret_cast<const float2*>(a.part_ml + (slot_of(p0 + i) * C::ROWS + row) * 2))
                                                       : make_float2(-INFINITY, 0.f);
                        };
                        float2 ml[BATCH];
                        float m = -INFINITY, l = 0.f;
                        for (int p0 = 0; p0 < parts; p0 += BATCH) {
                            load_ml(p0, ml);
                            float mn = m;
#pragma unroll
                            for (int i = 0; i < BATCH; ++i)
                                if (ml[i].y != 0.f) mn = fmaxf(mn, ml[i].x);  // (0: a part without a slot that this row sees)
                            l = l != 0.f ? l * fast_exp2(m - mn) : 0.f;
#pragma unroll
                            for (int i = 0; i < BATCH; ++i)
                                if (ml[i].y != 0.f) l = fmaf(ml[i].y, fast_exp2(ml[i].x - mn), l);
                            m = mn;
                        }
                        const float inv = 1.f / l;
                        uint16_t* orow = a.out + ((static_cast<size_t>(a.b0 + s.b) * a.n + tok) * a.Hq + s.h * a.G + (R - tok * a.G)) * D;
                        const int d_end = D / 4 * (part + 1) / of;
                        for (int d0 = D / 4 * part / of; d0 < d_end; d0 += 2) {
                            float4 acc[2] = {};
                            for (int p0 = 0; p0 < parts; p0 += BATCH) {
                                float4 o[BATCH][2];
                                if (parts > BATCH) load_ml(p0, ml);
#pragma unroll
                                for (int i = 0; i < BATCH; ++i)
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        if (p0 + i < parts && d0 + e < d_end)
                                            o[i][e] = __ldcg(reinterpret_cast<const float4*>(
                                                a.part_o + ((slot_of(p0 + i) * (D / 4) + d0 + e) * C::ROWS + row) * 4));
#pragma unroll
                                for (int i = 0; i < BATCH; ++i) {
                                    if (ml[i].y == 0.f) continue;
                                    const float w = fast_exp2(ml[i].x - m);
                                    // an infinity counts whatever its weight
                                    auto add = [&](float x, float y) { return w != 0.f ? fmaf(w, y, x) : isfinite(y) ? x : x + y; };
#pragma unroll
                                    for (int e = 0; e < 2; ++e)
                                        if (d0 + e < d_end)
                                            acc[e] = make_float4(add(acc[e].x, o[i][e].x), add(acc[e].y, o[i][e].y),
                                                                 add(acc[e].z, o[i][e].z), add(acc[e].w, o[i][e].w));
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (d0 + e < d_end)
                                    *reinterpret_cast<uint2*>(orow + 4 * (d0 + e)) =
                                        make_uint2(pack_bf16x2(acc[e].x * inv, acc[e].y * inv), pack_bf16x2(acc[e].z * inv, acc[e].w * inv));
                        }
                    }
                    __syncwarp();
                }
                // this warp leaves, and counts in what it did not do; the last one leaves the counter at 0
                if (lane == 0) {
                    const int add = 2 - did[slot];
                    if (atomicAdd(counter, add) + add == 2 * all) atomicExch(counter, 0);
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
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

template <int D, int NT>
cudaError_t configure() {
    using C = Cfg<D, NT>;
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, tree_decode_kernel<D, NT>);
    if (e != cudaSuccess) return e;
    // (the register split is only safe when the kernel is launched with exactly kLaunchRegs)
    if ((NT == 2 && attr.numRegs != kLaunchRegs) || attr.maxThreadsPerBlock < C::THREADS) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(tree_decode_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::ALLOC);
}

template <int D, int NT>
cudaError_t launch(const Shape& s, const TreeCall& c, const Args& args, cudaStream_t st) {
    using C = Cfg<D, NT>;
    Args a = args;
    a.groups = (c.n * a.G + C::ROWS - 1) / C::ROWS;
    // sequences of a launch: their tiles are counted in int
    const long long tiles = static_cast<long long>(s.n_kv_heads) * ((s.max_len + c.n + BN - 1) / BN);
    const int seqs = static_cast<int>(std::min<long long>(std::min(s.batch, kMaxSeqs), std::max((1LL << 30) / tiles, 1LL)));
    a.runs = static_cast<int>(std::min<long long>(std::max(c.num_sms / a.groups, 1), seqs * tiles));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.runs * a.groups));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::ALLOC;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    for (a.b0 = 0; a.b0 < s.batch; a.b0 += seqs) {
        a.batch = std::min(s.batch - a.b0, seqs);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, tree_decode_kernel<D, NT>, c.maps->k, c.maps->v, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t configure_tree_decode() {
    cudaError_t e = configure<128, 1>();
    if (e == cudaSuccess) e = configure<128, 2>();
    if (e == cudaSuccess) e = configure<64, 1>();
    if (e == cudaSuccess) e = configure<64, 2>();
    return e;
}

cudaError_t launch_tree_decode(const Shape& s, const TreeCall& c, cudaStream_t st) {
    Args a = {};
    a.q = c.q;
    a.k_new = c.k;
    a.v_new = c.v;
    a.d_hist = c.d_hist;
    a.parents = c.parents;
    a.k_cache = c.k_cache;
    a.v_cache = c.v_cache;
    a.cos_tab = c.cos_tab;
    a.sin_tab = c.sin_tab;
    a.out = c.out;
    a.part_o = c.part_o;
    a.part_ml = c.part_ml;
    a.counters = c.counters;
    a.err = c.err;
    a.wait_ns = c.wait_ns;
    a.scale_log2 = static_cast<float>(1.4426950408889634 / std::sqrt(static_cast<double>(s.head_dim)));
    a.n = c.n;
    a.Hq = s.n_q_heads;
    a.Hkv = s.n_kv_heads;
    a.G = s.n_q_heads / s.n_kv_heads;
    a.max_len = s.max_len;
    a.window = c.window;
    a.sinks = c.sinks;
    // a second tile of rows where one does not hold them all: it halves the passes over the keys
    const bool two = c.n * a.G > BM;
    if (s.head_dim == 128) return two ? launch<128, 2>(s, c, a, st) : launch<128, 1>(s, c, a, st);
    return two ? launch<64, 2>(s, c, a, st) : launch<64, 1>(s, c, a, st);
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
