"""The one bounded wait of the 4-bit decode, made to run out: what is affected is not written, the rest is right."""
import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U

pytestmark = pytest.mark.gpu

TIMEOUT = 2


# One new token: its two rows fall to the last two warps, while the warp that has their block has nothing else to do
# before it waits.  A block alone, the first of a run, the last of several pieces, items that whole CTAs take.
@pytest.mark.parametrize("B,Hkv,D,hist", [(1, 2, 128, 0), (1, 2, 64, 0), (1, 2, 128, 3000), (1, 1, 64, 5000), (12, 8, 128, 20),
                                          (12, 8, 64, 20), (12, 8, 128, 700)])
def test_outputs_of_a_wait_that_ran_out_are_not_written(B, Hkv, D, hist):
    import torch

    from paper_2607_15865_gb300.attention import Attention
    Hq, L = 2 * Hkv, hist + 1
    attn = Attention(B, Hq, Hkv, D, L, 1.0e4)
    tag = f"gave{B}{D}"
    ref = U.history(tag, B, Hkv, (L + 63) // 64 * 64, D, [hist] * B)
    q, k, v = U.new_tokens(tag, B, 1, Hq, Hkv, D)
    new = [U.dev_bf16(x) for x in (q, k, v)]
    lens = torch.full((B,), hist, dtype=torch.int32, device="cuda")
    before = U.copy(ref)
    tab, pos = K.tables(L, D, 1.0e4), np.array([hist])
    want, mass = np.zeros((2, B, 1, Hq, D))
    for b in range(B):
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
        want[b], mass[b] = K.attend(K.rope(q[b], pos, tab), pos, ref, b)
    attn.set_wait_limit(1)
    untouched = 0
    for _ in range(20):
        cache = U.to_dev(before, L)
        out = torch.full((B, 1, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        attn.kv4_decode(*new, lens, cache, out=out)
        code = attn.device_error()
        assert code in (0, TIMEOUT)
        U.same_cache(cache, ref, "cache")  # the new tokens are written all the same
        kept = (out == 7).reshape(B, Hkv, -1).all(-1).cpu().numpy()
        assert (kept.any() == (code == TIMEOUT)), f"error word {code}, {kept.sum()} items not written"
        wrote = np.broadcast_to(~kept[:, :, None, None], (B, Hkv, 2, D)).reshape(B, 1, Hq, D)
        some = torch.from_numpy(wrote.copy()).cuda()
        if wrote.any():
            U.close(out[some], want[wrote], mass[wrote], "items that did not wait too long")
        untouched += int(kept.sum())
    assert untouched > 0, "no wait ran out"
    attn.set_wait_limit(0)
    cache = U.to_dev(before, L)
    out = attn.kv4_decode(*new, lens, cache)
    assert attn.device_error() == 0
    U.close(out, want, mass, "with the default limit")
    U.same_cache(cache, ref, "with the default limit")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv,hist", [(2, 0), (2, 3000), (80, 600)])
def test_a_score_past_the_largest_float_is_nan_and_written(D, Hkv, hist):
    """Not to be taken for a part whose wait ran out: q and the new key are of the size of 2^64."""
    import torch

    from paper_2607_15865_gb300.attention import Attention
    attn = Attention(1, Hkv, Hkv, D, hist + 1, 1.0e4)
    ref = U.history(f"past{D}", 1, Hkv, (hist + 64) // 64 * 64, D, [hist])
    q, _, v = U.new_tokens(f"past{D}", 1, 1, Hkv, Hkv, D)
    q = K.f32_to_bf16(K.bf16_to_f64(q) * 2.0 ** 64)
    lens = torch.tensor([hist], dtype=torch.int32, device="cuda")
    out = torch.full((1, 1, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda")
    attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(q), U.dev_bf16(v), lens, U.to_dev(ref, hist + 1), out=out)
    assert attn.device_error() == 0 and out.isnan().all()
