"""kv4_prefill_kv asks for a workspace only where the call uses one."""
import ctypes

import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U

pytestmark = pytest.mark.gpu


def given(L, hist, n, Hq=8, Hkv=2, D=128):
    from paper_2607_15865_gb300.attention import Attention
    attn = Attention(1, Hq, Hkv, D, L, 1.0e4)
    ref = U.history("space", 1, Hkv, (L + 63) // 64 * 64, D, [hist])
    q, k, v = U.new_tokens("space", 1, n, Hq, Hkv, D)
    cache, new = U.to_dev(ref, L), [U.dev_bf16(x) for x in (q, k, v)]
    tab, pos = K.tables(L, D, 1.0e4), np.arange(hist, hist + n)
    ref.write(0, pos, K.rope(k[0], pos, tab), v[0])
    want, mass = K.attend(K.rope(q[0], pos, tab), pos, ref, 0)
    return attn, cache, new, ref, want[None], mass[None]


def test_a_few_tokens_over_a_long_history_allocate_their_output_alone():
    import torch
    hist, n = 8000, 3
    attn, cache, new, ref, want, mass = given(8100, hist, n)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = attn.kv4_prefill_kv(*new, hist, cache)
    assert torch.cuda.max_memory_allocated() - before <= 64 << 10  # the output is 6 KB, the workspace would be 8 MB
    U.close(out, want, mass, "no workspace")
    U.same_cache(cache, ref, "no workspace")


def test_the_c_call_without_a_workspace():
    """NULL where attn_kv4_prefill_workspace is 0, refused where it is not."""
    import torch

    from paper_2607_15865_gb300 import _lib
    hist, n = 100, 4
    attn, cache, new, ref, want, mass = given(300, hist, n)
    out = torch.zeros_like(new[0])
    p = [ctypes.c_void_p(t.data_ptr()) for t in new]
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def call(chunk):
        return attn.lib.attn_kv4_prefill_kv(attn._ctx, *p, hist, chunk, cache.ref, ctypes.c_void_p(out.data_ptr()), None, 0, st)

    assert attn.kv4_prefill_workspace(hist, n) == 0 and attn.kv4_prefill_workspace(hist, 60) == attn.kv4_workspace(160) > 0
    assert call(60) == _lib.ATTN_EINVAL
    torch.cuda.synchronize()
    assert not out.any()
    assert call(n) == _lib.ATTN_OK
    U.close(out, want, mass, "NULL")
    U.same_cache(cache, ref, "NULL")


def test_sizes():
    attn = given(300, 10, 1)[0]
    assert attn.kv4_prefill_workspace(0, 300) == attn.kv4_workspace(300) == 2 * 2 * 300 * 128 * 2
    assert [attn.kv4_prefill_workspace(*x) for x in ((0, 301), (-1, 4), (299, 2), (0, 0))] == [0] * 4
    assert [attn.kv4_workspace(n) for n in (0, 301)] == [0, 0]
