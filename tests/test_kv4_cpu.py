"""The 4-bit cache's format on the CPU: the oracle's own pins, the arithmetic the kernels rely on, refusals
that need no GPU."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv4_oracle as K

F = np.float32


def test_a_group_by_hand():
    # values -3 .. 4.5 in steps of 0.25 (31 of them) and a zero: (4.5 + 3) / 15 = 0.5 = s, z = 6
    x = np.concatenate([np.arange(-3.0, 4.75, 0.25), [0.0]])
    codes, scales = K.quantise(K.f32_to_bf16(x)[None])
    assert scales[0, 0] == 0x3F00 | 6
    # steps -6, -5.5, -5, -4.5, -4, ties to even: -6 -6 -5 -4 -4; 9 at the top; the zero is the zero point
    assert (codes[0, :5] == [0, 0, 1, 2, 2]).all() and codes[0, 30] == 15 and codes[0, 31] == 6


def test_packing_round_trip_and_order():
    c = np.arange(64, dtype=np.uint8).reshape(1, 64) % 16
    p = K.pack(c)
    assert (K.unpack(p) == c).all()
    w = int(p.view("<u4")[0, 0])
    assert [(w >> sh) & 15 for sh in K.BITS] == list(range(8))


def test_values_are_within_half_a_step_and_exactly_bf16():
    r = np.random.default_rng(1)
    x = r.normal(size=(500, 64)) * np.exp(r.normal(size=(500, 1)) * 3)
    x[::5] = np.abs(x[::5])
    bits = K.f32_to_bf16(x)
    codes, scales = K.quantise(bits)
    v = K.values(K.pack(codes), scales)
    K.f64_to_bf16_exact(v)
    s = np.repeat(K.bf16_to_f64(scales & np.uint16(0x7FF0)), 32, -1)
    # a value at either end may be a clamp away: rint(x / s) + z exceeds 15 by at most 1
    assert (np.abs(v - K.bf16_to_f64(bits)) <= s).all()
    assert np.mean(np.abs(v - K.bf16_to_f64(bits)) <= s / 2) > 0.99


def test_odd_groups_read_as_nan_and_empty_ones_as_zero():
    x = np.zeros((3, 32), np.uint16)
    x[1, 7], x[2, 9] = 0x7F80, 0x7FC0
    codes, scales = K.quantise(x)
    assert (codes == 0).all() and scales[0, 0] == 0x0080 and (scales[1:, 0] == K.NAN_SCALE).all()
    v = K.values(K.pack(codes), scales)
    assert (v[0] == 0).all() and np.isnan(v[1:]).all()


def test_float_quotient_by_reciprocal_is_exact():
    """kv4_round in float, as the kernels do it, against the rational quotient, for every pair of
    significands and every exponent that gives a code."""
    X = np.arange(128, 256)
    for S in range(8, 16):
        for k in range(-12, 5):
            x, s = F(X) * F(2.0) ** F(k), F(S)
            inv = F(1) / s
            t = x * inv
            t = (t + F(6144.0)) - F(6144.0)
            got = (t + F(12582912.0)) - F(12582912.0)
            want = [round(Fraction(int(v)) * Fraction(2) ** k / S) for v in X]  # Python rounds ties to even
            use = np.array([w <= 15 for w in want])
            assert (got[use] == np.array(want)[use]).all()


def test_float_quotient_by_one_fma_is_exact():
    """The same with the product and the first sum in one rounding, and on to the integer in one more."""
    X = np.arange(128, 256)
    for S in range(8, 16):
        for k in range(-12, 5):
            x, s = F(X) * F(2.0) ** F(k), F(S)
            inv = F(1) / s
            t = (x.astype(np.float64) * np.float64(inv) + 6144.0).astype(np.float32)  # exact in 64 bits before it rounds
            got = (t + F(12582912.0 - 6144.0)) - F(12582912.0)
            want = [round(Fraction(int(v)) * Fraction(2) ** k / S) for v in X]
            use = np.array([w <= 15 for w in want])
            assert (got[use] == np.array(want)[use]).all()
            t = (-x.astype(np.float64) * np.float64(inv) + 6144.0).astype(np.float32)
            got = (t + F(12582912.0 - 6144.0)) - F(12582912.0)
            assert (got[use] == -np.array(want)[use]).all()


def test_float_scale_is_exact():
    """kv4_scale_of in float against the rational definition, where (hi - lo) / 15 has 4 bits itself too."""
    r = np.random.default_rng(2)
    hi = K.bf16_to_f64(K.f32_to_bf16(np.abs(r.normal(size=20000))))
    lo = -K.bf16_to_f64(K.f32_to_bf16(np.abs(r.normal(size=20000)) * r.integers(0, 2, 20000)))
    hi[:4000] = 15 * r.integers(8, 16, 4000) * 2.0 ** r.integers(-8, 4, 4000) + lo[:4000]
    keep = (hi >= 0) & (K.bf16_to_f64(K.f32_to_bf16(hi)) == hi)
    hi, lo = hi[keep], lo[keep]
    lo[:50] = -(2.0 ** -30) * np.abs(lo[:50])  # under the rounding of hi - lo
    hi[:25] = 7.5
    q = (F(hi) * F(0.5) - F(lo) * F(0.5)) / F(7.5)
    up = (q.view(np.uint32) + np.uint32(0xFFFFF)) & np.uint32(0xFFF00000)
    up += (F(hi) * F(0.5) - up.view(np.float32) * F(7.5) > F(lo) * F(0.5)).astype(np.uint32) << np.uint32(20)
    got = np.maximum(up, np.uint32(0x00800000)).view(np.float32).astype(np.float64)
    for g, h, l in zip(got, hi, lo):
        d = (Fraction(h) - Fraction(l)) / 15
        assert Fraction(g) >= d
        m, e = np.frexp(g)
        below = np.ldexp(m * 16 - 1, e - 4) if m > 0.5 else np.ldexp(15.0, e - 5)  # the next smaller one
        if g > 2.0 ** -126:
            assert Fraction(float(below)) < d


def test_float_scale_from_a_low_quotient_is_exact():
    """The same with a product by a constant 1 to 2 parts in 2^22 below 1 / 7.5 in place of the quotient."""
    c = F(0.133333295)
    assert -2.0 < (float(c) * 7.5 - 1) * 2 ** 22 < -1.0
    r = np.random.default_rng(3)
    hi = K.bf16_to_f64(K.f32_to_bf16(np.abs(r.normal(size=20000)) * 2.0 ** r.integers(-20, 20, 20000)))
    lo = -K.bf16_to_f64(K.f32_to_bf16(np.abs(r.normal(size=20000)) * 2.0 ** r.integers(-20, 20, 20000)))
    lo[:6000] = 0
    hi[:3000] = 15 * r.integers(8, 16, 3000) * 2.0 ** r.integers(-8, 4, 3000)
    lo[3000:6000] = -15 * r.integers(8, 16, 3000) * 2.0 ** r.integers(-8, 4, 3000)
    lo[1500:3000] = -2.0 ** -30
    keep = (K.bf16_to_f64(K.f32_to_bf16(hi)) == hi) & (K.bf16_to_f64(K.f32_to_bf16(lo)) == lo)
    hi, lo = hi[keep], lo[keep]
    up = (((F(hi) * F(0.5) - F(lo) * F(0.5)) * c).view(np.uint32) + np.uint32(0xFFFFF)) & np.uint32(0xFFF00000)
    h, n = F(hi) * F(0.5), F(-lo) * F(0.5)
    up += (np.maximum(h, n) - up.view(np.float32) * F(7.5) > -np.minimum(h, n)).astype(np.uint32) << np.uint32(20)
    got = up.view(np.float32).astype(np.float64)
    for g, h, l in zip(got, hi, lo):
        d = (Fraction(h) - Fraction(l)) / 15
        m, e = np.frexp(g)
        below = np.ldexp(m * 16 - 1, e - 4) if m > 0.5 else np.ldexp(15.0, e - 5)
        assert Fraction(g) >= d > Fraction(float(below))


def test_refusals_without_a_context():
    from paper_2607_15865_gb300 import _lib, build
    build.build()
    lib = _lib.load()
    assert [lib.attn_kv4_slots(n) for n in (0, -1, 1, 64, 65, 8192, (1 << 20) + 1)] == [0, 0, 64, 64, 128, 8192, 0]
    c = _lib.AttnKv4(16, 16, 16, 16)
    ref, nul = ctypes.byref(c), None
    assert lib.attn_kv4_append(nul, 16, 16, 0, 1, ref, nul) == _lib.ATTN_EINVAL
    assert lib.attn_kv4_read(nul, ref, 0, 1, 16, 16, nul) == _lib.ATTN_EINVAL
    assert lib.attn_kv4_decode(nul, 16, 16, 16, 16, 1, ref, 16, nul) == _lib.ATTN_EINVAL
    assert lib.attn_kv4_prefill_kv(nul, 16, 16, 16, 0, 1, ref, 16, nul, 0, nul) == _lib.ATTN_EINVAL
    assert lib.attn_kv4_workspace(nul, 10) == 0


def test_a_cache_of_host_tensors_is_refused():
    import torch

    from paper_2607_15865_gb300.kv4 import Kv4Cache
    z = torch.zeros(1, 1, 64, 32, dtype=torch.uint8)
    with pytest.raises(TypeError):
        Kv4Cache(64, z, z, z, z)
