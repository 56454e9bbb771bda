"""Values of a new token that the 4-bit decode's products cannot hold reach the tokens that see it, and no other."""
import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,n", [(2, 4), (8, 5)])
@pytest.mark.parametrize("exp", [67, 72, 100, 125])
@pytest.mark.parametrize("route", ["decode", "prefill"])
def test_a_large_value_of_a_new_token_reaches_only_later_ones(D, Hq, n, exp, route):
    """Token 2's v is 2^exp times as large: tokens 0 and 1 come out as without it; so with its k."""
    import torch

    from paper_2607_15865_gb300.attention import Attention
    hist, L = 61, 100
    attn = Attention(1, Hq, 2, D, L, 1.0e4)
    tag = f"large{D}{Hq}"
    ref = U.history(tag, 1, 2, 128, D, [hist])
    q, k, v = U.new_tokens(tag, 1, n, Hq, 2, D)
    v[0, 2, 1] = K.f32_to_bf16(K.bf16_to_f64(v[0, 2, 1]) * 2.0 ** exp)
    k[0, 2, 0] = K.f32_to_bf16(K.bf16_to_f64(k[0, 2, 0]) * 2.0 ** exp)
    cache = U.to_dev(ref, L)
    new = [U.dev_bf16(x) for x in (q, k, v)]
    if route == "decode":
        out = attn.kv4_decode(*new, torch.tensor([hist], dtype=torch.int32, device="cuda"), cache)
    else:
        out = attn.kv4_prefill_kv(*new, hist, cache)
    tab, pos = K.tables(L, D, 1.0e4), np.arange(hist, hist + n)
    ref.write(0, pos, K.rope(k[0], pos, tab), v[0])
    U.same_cache(cache, ref, "cache")
    U.close(out[0, :2], *K.attend(K.rope(q[0, :2], pos[:2], tab), pos[:2], ref, 0), "earlier tokens")
