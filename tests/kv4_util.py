"""Inputs and bars of the 4-bit cache's tests.

Bars.  The packed cache is compared bit for bit: the quantiser is exact.  An output o of weights w and values
v, mass m = sum w |v| (sum w = 1): the kernels round each weight to bf16 (by at most 2^-8 of it), which moves
o by at most 2^-8 m and the sum it is divided by by 2^-8, and round the result (2^-8 |o|); float sums
and the exponential are orders below.  So |error| <= 2^-8 |o| + 2^-7 m, with 5% on top for those.
"""
from __future__ import annotations

import numpy as np

from oracle import kv4_oracle as K
from synthetic import gen

U16 = np.uint16


def bf16(tag, name, shape, sigma=1.0):
    return gen.normal_bf16(tag, name, shape, sigma)


def new_tokens(tag, B, n, Hq, Hkv, D):
    """q, k, v of n new tokens; keys with a few channels far from zero."""
    k = K.bf16_to_f64(bf16(tag, "k", (B, n, Hkv, D)))
    k[..., 3::17] += 3.0
    return bf16(tag, "q", (B, n, Hq, D), 1.3), K.f32_to_bf16(k), bf16(tag, "v", (B, n, Hkv, D))


def history(tag, B, Hkv, slots, D, hist):
    """A cache whose slots [0, hist[b]) hold tokens and whose others hold NaN groups with stray codes."""
    c = K.Cache(B, Hkv, slots, D)
    for t, name in enumerate("kv"):
        x = K.bf16_to_f64(bf16(tag, "hist_" + name, (B, Hkv, slots, D)))
        if name == "k":
            x[..., 3::17] += 3.0
        codes, scales = K.quantise(K.f32_to_bf16(x))
        c.codes[t][:] = K.pack(codes)
        c.scales[t][:] = scales
        for b in range(B):
            c.scales[t][b, :, hist[b]:] = K.NAN_SCALE
    return c


def copy(c):
    d = K.Cache.__new__(K.Cache)
    d.codes, d.scales = [x.copy() for x in c.codes], [x.copy() for x in c.scales]
    return d


def to_dev(c, max_len):
    """The cache as a Kv4Cache on the GPU."""
    import torch

    from paper_2607_15865_gb300.kv4 import Kv4Cache
    t = [torch.from_numpy(x.view(np.int16) if x.dtype == U16 else x).cuda() for x in
         (c.codes[0], c.scales[0], c.codes[1], c.scales[1])]
    return Kv4Cache(max_len, *t)


def same_cache(dev, c, what):
    for t, x in enumerate(((dev.k_codes, dev.k_scales), (dev.v_codes, dev.v_scales))):
        assert (x[0].cpu().numpy() == c.codes[t]).all(), f"{what}: {'kv'[t]} codes"
        assert (x[1].cpu().numpy().view(U16) == c.scales[t]).all(), f"{what}: {'kv'[t]} scales"


def dev_bf16(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def host_bits(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(U16)


def close(got, ref, mass, what):
    """got (a bf16 tensor) against the float64 ref; NaN exactly where ref has it."""
    g = K.bf16_to_f64(host_bits(got))
    assert (np.isnan(g) == np.isnan(ref)).all(), f"{what}: NaN in other places"
    ok = ~np.isnan(ref)
    err, bar = np.abs(g - ref)[ok], 1.05 * (2.0 ** -8 * np.abs(ref) + 2.0 ** -7 * mass)[ok]
    rel = np.linalg.norm(err) / max(np.linalg.norm(ref[ok]), 1e-300)
    print(f"[parity] {what}: rel {rel:.3e}, worst of bar {(err / np.maximum(bar, 1e-300)).max():.3f}")
    assert (err <= bar).all(), f"{what}: {(err / np.maximum(bar, 1e-300)).max():.2f} of the bar"
