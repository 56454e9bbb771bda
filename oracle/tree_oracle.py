"""Attention under a sliding window with sinks, of chains and trees of new tokens, and the move of accepted tokens, in
numpy float64: straight from the definitions in include/attn.h; shares nothing with the library.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.kv4_oracle import bf16_to_f64, f32_to_bf16, rope, tables  # noqa: F401  (the rotation every stage uses)

GONE = -2  # a parent that says that there is no token


def kin(parents):
    """Per token its ancestors and itself, in order ([] where there is no token); None where it is no tree."""
    chains = []
    for i, p in enumerate(parents):
        if p < GONE or p >= i or (p >= 0 and not chains[p]):
            return None
        chains.append([] if p == GONE else (chains[p] if p >= 0 else []) + [i])
    return chains


def chain(n):
    return list(range(-1, n - 1))


def seen_slots(hist, chains, i, window, sinks):
    """Slots that token i sees, ascending; window None: all that it may."""
    at = {hist + j: hist + len(chains[j]) - 1 for j in chains[i]}  # slot -> position
    p = hist + len(chains[i]) - 1
    ok = lambda t: window is None or p - t < window or t < sinks  # noqa: E731
    if window is None:
        old = list(range(hist))
    else:
        lo = max(0, p - window + 1)
        old = list(range(min(sinks, lo, hist))) + list(range(min(lo, hist), hist))
    return old + [s for s, t in at.items() if ok(t)]


def attend(q, k, v, hist, parents, kc, vc, tab, window=None, sinks=0):
    """One sequence: q [n, Hq, D], k, v [n, Hkv, D], kc, vc [Hkv, L, D] bf16 bits (written in place), parents a list.
    -> out, mass [n, Hq, D] float64 (NaN where there is no token), or None where the sequence is skipped."""
    chains = kin(parents)
    L = kc.shape[1]
    if chains is None or not 0 <= hist <= L:
        return None
    live = [i for i, c in enumerate(chains) if c]
    if live and hist + live[-1] >= L:
        return None
    for i in live:
        kc[:, hist + i] = rope(k[i:i + 1], np.array([hist + len(chains[i]) - 1]), tab)[0]
        vc[:, hist + i] = v[i]
    n, hq, d = q.shape
    G = hq // kc.shape[0]
    out, mass = np.full((2, n, hq, d), np.nan)
    for i in live:
        qr = bf16_to_f64(rope(q[i:i + 1], np.array([hist + len(chains[i]) - 1]), tab)[0])
        slots = seen_slots(hist, chains, i, window, sinks)
        for g in range(kc.shape[0]):
            kk, vv = bf16_to_f64(kc[g, slots]), bf16_to_f64(vc[g, slots])
            with np.errstate(invalid="ignore", over="ignore"):
                a = qr[g * G:(g + 1) * G] @ kk.T / math.sqrt(d)
                w = np.exp(a - a.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[i, g * G:(g + 1) * G], mass[i, g * G:(g + 1) * G] = w @ vv, w @ np.abs(vv)
    return out, mass


def accept(hist, parents, leaf, caches):
    """One sequence: caches a list of [Hkv, L, D] arrays (changed in place) -> the new length."""
    chains = kin(parents)
    if chains is None or not -1 <= leaf < len(parents) or (leaf >= 0 and not chains[leaf]):
        return hist
    live = [i for i, c in enumerate(chains) if c]
    if not 0 <= hist <= caches[0].shape[1] or (live and hist + live[-1] >= caches[0].shape[1]):
        return hist
    path = chains[leaf] if leaf >= 0 else []
    for x in caches:
        x[:, hist:hist + len(path)] = x[:, [hist + i for i in path]]
    return hist + len(path)
