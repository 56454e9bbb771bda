"""Every slot counts, and counts once: the 4-bit decode with q = 0, where an output is the mean of the values seen.

Values mark their place: in the first half of D by block of 32 slots, in the second by slot, and their size by sequence
and head.  The weights are equal, so that rounding them cancels in the quotient: the bar is the rounding of the output (2^-8
of it, 5% on top) and 2^-16 for float sums.  test_the_bar_tells_a_lost_block (on the CPU) plants mistakes in the
expected values."""
import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U


def ramp(B, top):
    return [top * ((i * 7) % B) // (B - 1) for i in range(B)]


def marked(factor, slots, D):
    """bf16 bits [slots, D] of a head's values."""
    p, h = np.arange(slots)[:, None], D // 2
    d = np.arange(h)[None]
    x = np.concatenate([p // 32 % h == d, p % h == d], 1) * float(factor)
    return K.f32_to_bf16(x)


def factor_of(b, g):
    return 1 + (3 * b + g) % 7


def means(D, b, g, counts):
    """The means over the first n slots, for n in counts: float64 [len(counts), D]."""
    codes, scales = K.quantise(marked(factor_of(b, g), max(counts), D))
    total = np.cumsum(K.values(K.pack(codes), scales), 0)
    return np.stack([total[n - 1] / n for n in counts])


def bar(want):
    return 1.05 * 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * np.abs(want).max(-1, keepdims=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [33, 500, 2001, 8191])
def test_the_bar_tells_a_lost_block(D, n):
    codes, scales = K.quantise(marked(1, n, D))
    v = K.values(K.pack(codes), scales)
    want = v.mean(0)
    for first, count, times in ((0, 32, 0), (n - 1, 1, 0), (32 * (n // 64), 32, 2), (n // 2, 16, 0), (n // 3, 1, 2)):
        w = np.ones(n)
        w[first:first + count] = times
        got = w @ v / w.sum()
        if not got.any() or (D == 64 and n > 8000 and count == 1):
            continue  # a slot of 8191 in 32 places is 2^-8 of its place
        assert (np.abs(got - want) > 1.5 * bar(want)).any(), f"slots {first} .. {first + count - 1} {times} times"


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,hist,n", [
    # one sequence: whole, in pieces
    (1, 8, 2, 128, [700], 1), (1, 8, 2, 64, [1500], 1), (1, 8, 2, 128, [8190], 1), (1, 40, 8, 128, [5999], 1),
    (1, 1, 1, 64, [8999], 1), (1, 32, 8, 128, [8188], 4), (1, 16, 1, 128, [4100], 9), (1, 5, 5, 64, [3333], 16),
    # several in pieces in proportion
    (6, 8, 2, 128, ramp(6, 1499), 1), (31, 2, 1, 64, ramp(31, 2890), 3), (9, 4, 2, 128, [3999, 17, 2048, 0, 1000, 3500, 33, 64, 1], 1),
    (2, 32, 8, 64, [4001, 1234], 5),
    # equal runs
    (12, 16, 8, 128, ramp(12, 1299), 1), (12, 16, 8, 64, ramp(12, 2400), 1), (12, 16, 8, 128, ramp(12, 690), 8),
    (20, 32, 8, 64, ramp(20, 600), 4), (16, 32, 8, 128, ramp(16, 2183), 1), (3, 64, 64, 128, [900, 31, 320], 1),
    # whole items
    (40, 8, 4, 128, [200] * 40, 1), (40, 8, 4, 64, [(37 * i) % 290 for i in range(40)], 5), (64, 8, 8, 128, [400] * 64, 1),
    # several launches
    (130, 2, 1, 64, ramp(130, 449), 1), (129, 4, 2, 128, ramp(129, 170), 2),
])
def test_every_slot_counts_once(B, Hq, Hkv, D, hist, n):
    import torch

    from paper_2607_15865_gb300.attention import Attention
    L = max(hist) + n
    slots = (L + 63) // 64 * 64
    attn = Attention(B, Hq, Hkv, D, L, 1.0e4)
    r = np.random.default_rng(7)
    ref = K.Cache(B, Hkv, slots, D)
    ref.codes[0][:] = r.integers(0, 256, ref.codes[0].shape, dtype=np.uint8)  # any finite keys
    ref.scales[0][:] = r.integers(0x3E00, 0x4000, ref.scales[0].shape, dtype=np.uint16)
    v = np.zeros((B, n, Hkv, D), np.uint16)
    packed = {}
    for b in range(B):
        for g in range(Hkv):
            f = factor_of(b, g)
            if f not in packed:
                bits = marked(f, slots, D)
                codes, scales = K.quantise(bits)
                packed[f] = K.pack(codes), scales, bits
            ref.codes[1][b, g, :hist[b]] = packed[f][0][:hist[b]]
            ref.scales[1][b, g] = K.NAN_SCALE
            ref.scales[1][b, g, :hist[b]] = packed[f][1][:hist[b]]
            v[b, :, g] = packed[f][2][hist[b]:hist[b] + n]
    k = U.bf16("blocks", "k", (B, n, Hkv, D))
    lens = torch.tensor(hist, dtype=torch.int32, device="cuda")
    out = attn.kv4_decode(U.dev_bf16(np.zeros((B, n, Hq, D), np.uint16)), U.dev_bf16(k), U.dev_bf16(v), lens, U.to_dev(ref, L))
    assert attn.device_error() == 0
    got = K.bf16_to_f64(U.host_bits(out))
    for b in range(B):
        for g in range(Hkv):
            want = means(D, b, g, [hist[b] + i + 1 for i in range(n)])[:, None]
            err = np.abs(got[b, :, g * (Hq // Hkv):(g + 1) * (Hq // Hkv)] - want)
            assert (err <= bar(want)).all(), f"sequence {b}, kv head {g}: {(err / np.maximum(bar(want), 1e-300)).max():.2f} of the bar"


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,D,hist,n", [
    (1, 8, 2, 128, [8191], 1), (1, 8, 2, 64, [8191], 1), (2, 8, 1, 64, [8999, 4444], 1), (1, 32, 8, 128, [8188], 4),
    (4, 8, 2, 128, [6000, 100, 1500, 3000], 3), (16, 32, 8, 128, ramp(16, 1800), 1), (12, 16, 8, 64, ramp(12, 1990), 4),
])
def test_error_norms(B, Hq, Hkv, D, hist, n):
    """A weight and an output are rounded to bf16, each to within 2^-8 and so by at most 2^-8 / sqrt 3 = 0.00226 rms; values of random
    sign carry the first over to the output as they carry the output itself: 0.0032 together.  So 0.004 of the norm of
    all outputs; half as much again for the D of a row, whose quotient of norms varies."""
    import torch

    from paper_2607_15865_gb300.attention import Attention
    L = max(hist) + n
    attn = Attention(B, Hq, Hkv, D, L, 1.0e4)
    tag = f"norm{B}{D}"
    ref = U.history(tag, B, Hkv, (L + 63) // 64 * 64, D, hist)
    q, k, v = U.new_tokens(tag, B, n, Hq, Hkv, D)
    lens = torch.tensor(hist, dtype=torch.int32, device="cuda")
    out = attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), lens, U.to_dev(ref, L))
    assert attn.device_error() == 0
    tab, want = K.tables(L, D, 1.0e4), np.zeros(out.shape)
    for b, h in enumerate(hist):
        pos = np.arange(h, h + n)
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
        want[b] = K.attend(K.rope(q[b], pos, tab), pos, ref, b)[0]
    err = K.bf16_to_f64(U.host_bits(out)) - want
    rows = np.linalg.norm(err, axis=-1) / np.linalg.norm(want, axis=-1)
    whole = np.linalg.norm(err) / np.linalg.norm(want)
    print(f"[parity] all {whole:.2e}, worst row {rows.max():.2e}")
    assert whole <= 0.004 and rows.max() <= 0.006
