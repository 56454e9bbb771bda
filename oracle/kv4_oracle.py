"""The 4-bit KV cache in numpy float64: quantiser, packed format, RoPE and attention over it.

Straight from the definition in include/attn.h (attn_kv4); shares nothing with the library.
Float64 holds every step of the quantiser exactly: a bf16's 8 bits, sums of two of them (but for
the range of a group whose extremes are 2^45 apart, which is compared as such), and quotients
that are compared with half-integers at least 2^-10 away or met exactly.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
BITS = (0, 16, 4, 20, 8, 24, 12, 28)
NAN_SCALE = 0x7FF0


def bf16_to_f64(bits):
    return (np.asarray(bits, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)


def f32_to_bf16(x):
    """float32 -> bf16 bits, nearest even (NaN stays NaN)."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def f64_to_bf16_exact(x):
    """Bits of values that are bf16 numbers (or NaN)."""
    f = np.asarray(x, dtype=np.float64).astype(np.float32)
    bits = f.view(np.uint32)
    assert ((bits & 0xFFFF) == 0)[~np.isnan(f)].all(), "not a bf16"
    return (bits >> 16).astype(np.uint16)


def quantise(bits):
    """bf16 bits [..., D] -> codes 0..15 uint8 [..., D], scales uint16 [..., D / 32]."""
    x = bf16_to_f64(bits).reshape(bits.shape[:-1] + (-1, GROUP))
    finite = np.isfinite(x).all(-1)
    x = np.where(finite[..., None], x, 0.0)
    lo, hi = np.minimum(x.min(-1), 0.0), np.maximum(x.max(-1), 0.0)
    m, e = np.frexp((hi - lo) / 15.0)  # m in [0.5, 1)
    m = np.ceil(m * 16.0)
    # where hi - lo drops one extreme beside the other: the larger less 15 s is exact
    m += np.maximum(hi, -lo) - 15.0 * np.ldexp(m, e - 4) > -np.minimum(hi, -lo)
    s = np.maximum(np.ldexp(m, e - 4), 2.0 ** -126)
    z = np.rint(-lo / s)
    c = np.clip(np.rint(x / s[..., None]) + z[..., None], 0, 15)
    scales = np.where(finite, f64_to_bf16_exact(s) | z.astype(np.uint16), np.uint16(NAN_SCALE))
    c = np.where(finite[..., None], c, 0.0).astype(np.uint8)
    return c.reshape(bits.shape), scales.astype(np.uint16)


def pack(codes):
    """Codes [..., D] -> packed bytes uint8 [..., D / 2]."""
    c = codes.reshape(codes.shape[:-1] + (-1, 8)).astype(np.uint32)
    w = np.zeros(c.shape[:-1], dtype="<u4")
    for j, sh in enumerate(BITS):
        w |= c[..., j] << np.uint32(sh)
    return w.view(np.uint8).reshape(codes.shape[:-1] + (-1,))


def unpack(packed):
    w = np.ascontiguousarray(packed).view("<u4")
    return np.stack([(w >> np.uint32(sh)) & np.uint32(15) for sh in BITS], -1).astype(np.uint8).reshape(
        packed.shape[:-1] + (2 * packed.shape[-1],))


def values(packed, scales):
    """The float64 values [..., D] of packed bytes and scales."""
    c = unpack(packed).astype(np.float64)
    m = np.asarray(scales, dtype=np.uint16)
    s, z = bf16_to_f64(m & np.uint16(0x7FF0)), (m & np.uint16(15)).astype(np.float64)
    return (c - np.repeat(z, GROUP, -1)) * np.repeat(s, GROUP, -1)


def tables(max_len, head_dim, theta):
    inv = np.array([theta ** (-2.0 * j / head_dim) for j in range(head_dim // 2)])
    ang = np.arange(max_len, dtype=np.float64)[:, None] * inv
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def rope(bits, pos, tab):
    """bf16 bits [..., n, H, D] at positions pos [..., n] -> rotated bf16 bits: float arithmetic, each
    product and the difference or sum rounded, then rounded to bf16."""
    x = (np.asarray(bits, dtype=np.uint32) << 16).view(np.float32)
    h = x.shape[-1] // 2
    cos, sin = (t[pos][..., None, :] for t in tab)
    a, b = x[..., :h], x[..., h:]
    with np.errstate(invalid="ignore", over="ignore"):
        return f32_to_bf16(np.concatenate([a * cos - b * sin, b * cos + a * sin], -1))


class Cache:
    """A batch's 4-bit cache on the host: packed codes and scales, updated in place."""

    def __init__(self, batch, n_kv_heads, slots, head_dim):
        self.codes = [np.zeros((batch, n_kv_heads, slots, head_dim // 2), np.uint8) for _ in "kv"]
        self.scales = [np.zeros((batch, n_kv_heads, slots, head_dim // GROUP), np.uint16) for _ in "kv"]

    def write(self, b, pos, k_rot, v):
        """k_rot (rotated), v: bf16 bits [n, Hkv, D] of sequence b at slots pos."""
        for t, x in enumerate((k_rot, v)):
            c, s = quantise(x)
            self.codes[t][b][:, pos] = pack(c).swapaxes(0, 1)
            self.scales[t][b][:, pos] = s.swapaxes(0, 1)

    def values(self, b, g, n):
        return tuple(values(self.codes[t][b, g, :n], self.scales[t][b, g, :n]) for t in range(2))


def attend(q_rot, pos, cache, b):
    """q_rot: bf16 bits [n, Hq, D] at slots pos of sequence b -> (out, mass): the attention output and the same
    weighted mean of |v|, float64 [n, Hq, D]."""
    n, hq, d = q_rot.shape
    hkv = cache.codes[0].shape[1]
    q = bf16_to_f64(q_rot)
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    for g in range(hkv):
        k, v = cache.values(b, g, int(pos[-1]) + 1)
        for i in range(n):
            p = int(pos[i]) + 1  # slots this token sees
            with np.errstate(invalid="ignore", over="ignore"):
                a = q[i, g * (hq // hkv):(g + 1) * (hq // hkv)] @ k[:p].T / math.sqrt(d)
                w = np.exp(a - a.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[i, g * (hq // hkv):(g + 1) * (hq // hkv)] = w @ v[:p]
                mass[i, g * (hq // hkv):(g + 1) * (hq // hkv)] = w @ np.abs(v[:p])
    return out, mass
