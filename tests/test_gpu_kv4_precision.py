"""The 4-bit decode at head_dim 64 holds its softmax weights to 2^-16, in two bf16 parts.

Bar: the output's own rounding to bf16, 2^-8 |o| at most, with 5% on top, and 2^-12 of the weighted mean of
|v|: 2^-15 for weights that are off by 2^-16 and for their sum, the rest for the float scores (a few 2^-24 of sums of some
hundreds before the scale of 1/8, so up to 2^-14 in a weight and in the sum).  One rounding of the weights to bf16 moves the
outputs by up to 2^-8 of that mean, wherever few slots share the weight.
"""
import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def within(got, ref, mass, what):
    g = K.bf16_to_f64(U.host_bits(got))
    err, bar = np.abs(g - ref), 1.05 * 2.0 ** -8 * np.abs(ref) + 2.0 ** -12 * mass
    assert (err <= bar).all(), f"{what}: {(err / np.maximum(bar, 1e-300)).max():.2f} of the bar"


@pytest.mark.parametrize("Hq,Hkv,hist,n", [
    (8, 2, [1, 2, 5, 40], 1),       # pieces of one part
    (8, 2, [1500, 33], 1),          # and of several
    (8, 2, [3, 700], 4),            # 16 columns
    (14, 2, [300, 9, 2], 3),        # two groups of columns
    (16, 8, [i % 50 for i in range(30)], 1),    # runs
    (16, 8, [7 * i % 300 for i in range(30)], 5),
    (16, 8, [11 * i % 100 for i in range(12)], 8),
])
def test_decode(Hq, Hkv, hist, n):
    import torch

    from paper_2607_15865_gb300.attention import Attention
    B, D, L = len(hist), 64, max(hist) + n
    attn = Attention(B, Hq, Hkv, D, L, 1.0e4)
    tag = f"fine{Hq}{n}{B}"
    ref = U.history(tag, B, Hkv, (L + 63) // 64 * 64, D, hist)
    q, k, v = U.new_tokens(tag, B, n, Hq, Hkv, D)
    lens = torch.tensor(hist, dtype=torch.int32, device="cuda")
    out = attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), lens, U.to_dev(ref, L))
    tab = K.tables(L, D, 1.0e4)
    for b, h in enumerate(hist):
        pos = np.arange(h, h + n)
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
        within(out[b], *K.attend(K.rope(q[b], pos, tab), pos, ref, b), f"sequence {b}")
    assert attn.device_error() == 0


def test_prefill_of_a_few_tokens():
    """The same kernel behind kv4_prefill_kv."""
    from paper_2607_15865_gb300.attention import Attention
    L, D, hist, n = 60, 64, 17, 4
    attn = Attention(1, 8, 2, D, L, 1.0e4)
    ref = U.history("finep", 1, 2, 64, D, [hist])
    q, k, v = U.new_tokens("finep", 1, n, 8, 2, D)
    out = attn.kv4_prefill_kv(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), hist, U.to_dev(ref, L))
    tab, pos = K.tables(L, D, 1.0e4), np.arange(hist, hist + n)
    ref.write(0, pos, K.rope(k[0], pos, tab), v[0])
    within(out[0], *K.attend(K.rope(q[0], pos, tab), pos, ref, 0), "chunk")
