"""Inputs and bars of the tests of windows and trees.

Bars.  An output o of weights w and values v, mass m = sum w |v| (sum w = 1): the kernels round each weight to bf16, by at
most 2^-8 of it, in the products with v, which moves o by at most 2^-8 m, and round the result (2^-8 |o|); the sum that it
is divided by is of the unrounded weights.  Float sums and the exponential are orders below: 5% on top for those.
The caches are compared bit for bit: RoPE is float arithmetic, each step rounded, on both sides.
"""
from __future__ import annotations

import numpy as np

from oracle import tree_oracle as T
from synthetic import gen

NAN = np.uint16(0x7FC0)
THETA = 1.0e4


def bf16(tag, name, shape, sigma=1.0):
    return gen.normal_bf16(tag, name, shape, sigma)


def new_tokens(tag, B, n, Hq, Hkv, D):
    """q, k, v of n new tokens; keys with a few channels far from zero."""
    k = T.bf16_to_f64(bf16(tag, "k", (B, n, Hkv, D)))
    k[..., 3::17] += 3.0
    return bf16(tag, "q", (B, n, Hq, D), 1.3), T.f32_to_bf16(k), bf16(tag, "v", (B, n, Hkv, D))


def history(tag, B, Hkv, L, D, lens):
    """Caches whose slots [0, lens[b]) hold tokens and whose others hold NaN."""
    out = []
    for name in "kv":
        x = T.bf16_to_f64(bf16(tag, "hist_" + name, (B, Hkv, L, D)))
        if name == "k":
            x[..., 3::17] += 3.0
        x = T.f32_to_bf16(x)
        for b in range(B):
            x[b, :, max(lens[b], 0):] = NAN
        out.append(x)
    return out


def random_tree(seed, n, width, gone=0, roots=0.1):
    """Parents of n tokens, the last `gone` of them absent."""
    r = np.random.default_rng([seed, n, width])
    p = [-1 if i == 0 or r.random() < roots else int(r.integers(max(0, i - width), i)) for i in range(n)]
    return [T.GONE if i >= n - gone else x for i, x in enumerate(p)]


def dev(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def dev_i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bits(t):
    import torch
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


def want(new, lens, parents, kc, vc, L, window=None, sinks=0):
    """The oracle over a batch, caches written in place: out, mass (NaN: a row that is not written)."""
    q, k, v = new
    tab = T.tables(L, q.shape[-1], THETA)
    out, mass = np.full((2, *q.shape), np.nan)
    for b in range(q.shape[0]):
        got = T.attend(q[b], k[b], v[b], lens[b], parents[b], kc[b], vc[b], tab, window, sinks)
        if got is not None:
            out[b], mass[b] = got
    return out, mass


def rows_written(lens, parents, L):
    """[B, n]: the rows of out that a call writes."""
    rows = []
    for h, p in zip(lens, parents):
        c = T.kin(p)
        live = [bool(x) for x in c] if c is not None else [False] * len(p)
        last = max((i for i, x in enumerate(live) if x), default=-1)
        rows.append(live if c is not None and 0 <= h <= L and h + last < L else [False] * len(p))
    return np.array(rows)


def close(got, ref, mass, what, rows=None):
    """got (a bf16 tensor) against the float64 ref in the given rows; NaN and infinities exactly where ref has them."""
    g = T.bf16_to_f64(bits(got))
    if rows is not None:
        g, ref, mass = g[rows], ref[rows], mass[rows]
    assert (np.isnan(g) == np.isnan(ref)).all(), f"{what}: NaN in other places"
    inf = np.isinf(ref)
    assert (g[inf] == ref[inf]).all() and not np.isinf(g[~inf]).any(), f"{what}: infinities in other places"
    ok = np.isfinite(ref)
    err, bar = np.abs(g[ok] - ref[ok]), 1.05 * 2.0 ** -8 * (np.abs(ref[ok]) + mass[ok])
    if err.size:
        rel = np.linalg.norm(err) / max(np.linalg.norm(ref[ok]), 1e-300)
        print(f"[parity] {what}: rel {rel:.3e}, worst of bar {(err / np.maximum(bar, 1e-300)).max():.3f}")
        assert (err <= bar).all(), f"{what}: {(err / np.maximum(bar, 1e-300)).max():.2f} of the bar"


def same_k(got, ref):
    """Bit for bit, but for which NaN a rotated NaN is."""
    g = bits(got)
    return ((g == ref) | (np.isnan(T.bf16_to_f64(g)) & np.isnan(T.bf16_to_f64(ref)))).all()


def check(attn, new, lens, parents, window, sinks, tag, kc=None, vc=None, expect_err=0, call=None):
    """One call against the oracle: outputs, caches bit for bit, rows that are not written, the error word.
    parents: per sequence a list, or None for chains (window_decode)."""
    import torch
    B, n = new[0].shape[:2]
    L = attn.max_len
    if kc is None:
        kc, vc = history(tag, B, attn.n_kv_heads, L, attn.head_dim, lens)
    gk, gv = dev(kc), dev(vc)
    rk, rv = kc.copy(), vc.copy()
    tree = [T.chain(n)] * B if parents is None else parents
    ref, mass = want(new, lens, tree, rk, rv, L, window or None, sinks)
    out = torch.full((B, n, attn.n_q_heads, attn.head_dim), 7.0, dtype=torch.bfloat16, device="cuda")
    args = [dev(x) for x in new]
    if call is not None:
        call(args, gk, gv, out)
    elif parents is None:
        attn.window_decode(*args, dev_i32(lens), window, gk, gv, sinks=sinks, out=out)
    else:
        attn.tree_decode(*args, dev_i32(lens), dev_i32(parents), gk, gv, window=window, sinks=sinks, out=out)
    assert attn.device_error() == expect_err
    rows = rows_written(lens, tree, L)
    close(out, ref, mass, tag, rows)
    assert (out.float().cpu().numpy()[~rows] == 7.0).all(), f"{tag}: rows of no token were written"
    assert same_k(gk, rk), f"{tag}: k cache"
    assert (bits(gv) == rv).all(), f"{tag}: v cache"
    return out
