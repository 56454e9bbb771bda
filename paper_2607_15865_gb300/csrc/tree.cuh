// tree.cuh -- the relations of a tree of drafted tokens, and which slots a query sees.
//
// parents[i] of token i: the index of another token before it, -1 where it follows the history, -2 where there is no
// token i.  kin(i): i and its ancestors, a bit each; its depth, from 0, is one less than their number.
// A query at position p sees slot s of a token at position t(s) iff the slot is the history's or its kin's and
//   t(s) <= p and (p - t(s) < window or t(s) < sinks).
#pragma once

#include "internal.h"

namespace attn {

constexpr int kMaxTree = 64;  // tokens of a tree: a bit each of a 64-bit word

__device__ __forceinline__ uint64_t shfl64(uint64_t v, int lane) {
    const uint32_t lo = __shfl_sync(0xFFFFFFFFu, static_cast<uint32_t>(v), lane);
    const uint32_t hi = __shfl_sync(0xFFFFFFFFu, static_cast<uint32_t>(v >> 32), lane);
    return static_cast<uint64_t>(hi) << 32 | lo;
}

// The kin of tokens `lane` and `lane` + 32 of n <= 64 (0: no such token), a converged warp.  parents NULL: a chain.  Returns the tokens
// up to the last that there is, or -1 where a parent is not a token before its child.  By pointer doubling: after r rounds kin
// holds the ancestors up to 2^r steps away and up the one that is 2^r steps away.
__device__ __forceinline__ int tree_kin(const int32_t* parents, int n, int lane, uint64_t (&kin)[2]) {
    if (parents == nullptr) {
        kin[0] = lane < n ? (2ull << lane) - 1 : 0;
        kin[1] = lane + 32 < n ? (2ull << (lane + 32)) - 1 : 0;  // (2 << 63 is 0, less 1 all bits)
        return n;
    }
    int up[2];
    bool bad = false;
    uint64_t there = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        up[h] = i < n ? __ldg(parents + i) : -2;
        bad |= up[h] < -2 || up[h] >= i;
        there |= static_cast<uint64_t>(__ballot_sync(0xFFFFFFFFu, up[h] >= -1)) << (32 * h);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        kin[h] = up[h] >= -1 ? 1ull << i : 0;
        bad |= up[h] >= 0 && up[h] < i && !(there >> up[h] & 1);
    }
    if (__any_sync(0xFFFFFFFFu, bad)) return -1;
#pragma unroll 1
    for (int far = 1; far < n; far *= 2) {
        uint64_t k[2];
        int u[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int from = up[h] & 31;
            const uint64_t k0 = shfl64(kin[0], from), k1 = shfl64(kin[1], from);
            const int u0 = __shfl_sync(0xFFFFFFFFu, up[0], from), u1 = __shfl_sync(0xFFFFFFFFu, up[1], from);
            k[h] = up[h] < 0 ? 0 : up[h] < 32 ? k0 : k1;
            u[h] = up[h] < 0 ? up[h] : up[h] < 32 ? u0 : u1;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            kin[h] |= k[h];
            up[h] = u[h];
        }
    }
    return 64 - __clzll(static_cast<long long>(there));
}

}  // namespace attn
