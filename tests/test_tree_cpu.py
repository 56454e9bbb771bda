"""Windows and trees without a GPU: what pins the oracle, and what the C calls refuse before any CUDA call."""
import ctypes

import numpy as np
import pytest

from oracle import kv4_oracle as K
from oracle import tree_oracle as T
from tests import tree_util as U


@pytest.fixture(scope="module")
def lib():
    from paper_2607_15865_gb300 import _lib, build
    build.build()
    return _lib.load()


def test_kin():
    assert T.kin([-1, 0, 0, 2, -1, 4]) == [[0], [0, 1], [0, 2], [0, 2, 3], [4], [4, 5]]
    assert T.kin([-1, -2, 0, -2]) == [[0], [], [0, 2], []]
    assert T.kin(T.chain(4)) == [[0], [0, 1], [0, 1, 2], [0, 1, 2, 3]]
    for bad in ([0], [-1, 1], [-1, 2, 0], [-3], [-2, 0], [-1, 64]):
        assert T.kin(bad) is None


def test_seen_slots_by_hand():
    c = T.kin([-1, 0, 0, 2])
    assert T.seen_slots(3, c, 3, None, 0) == [0, 1, 2, 3, 5, 6]
    assert T.seen_slots(3, c, 3, 3, 0) == [3, 5, 6]       # positions 3, 4, 5
    assert T.seen_slots(3, c, 3, 4, 1) == [0, 2, 3, 5, 6]
    assert T.seen_slots(3, c, 3, 1, 0) == [6]
    assert T.seen_slots(3, c, 3, 1, 100) == [0, 1, 2, 3, 5, 6]
    assert T.seen_slots(0, c, 3, 2, 1) == [0, 2, 3]        # the first drafted token is position 0: a sink
    chain = T.kin(T.chain(3))
    for i in range(3):
        for w in range(1, 9):
            for s in range(9):
                p = 5 + i
                assert T.seen_slots(5, chain, i, w, s) == [x for x in range(p + 1) if p - x < w or x < s]


def test_a_chain_without_a_window_is_the_causal_oracle():
    """One head group against the attention oracle's own float64 sum over a causal cache."""
    n, Hq, Hkv, D, hist, L = 3, 4, 2, 64, 11, 20
    q, k, v = U.new_tokens("pin", 1, n, Hq, Hkv, D)
    kc, vc = U.history("pin", 1, Hkv, L, D, [hist])
    tab = T.tables(L, D, U.THETA)
    out, _ = T.attend(q[0], k[0], v[0], hist, T.chain(n), kc[0], vc[0], tab)
    pos = np.arange(hist, hist + n)
    kk = np.concatenate([K.bf16_to_f64(kc[0, :, :hist]), K.bf16_to_f64(K.rope(k[0], pos, tab)).swapaxes(0, 1)], 1)
    vv = np.concatenate([K.bf16_to_f64(vc[0, :, :hist]), K.bf16_to_f64(v[0]).swapaxes(0, 1)], 1)
    qr = K.bf16_to_f64(K.rope(q[0], pos, tab))
    for i in range(n):
        for h in range(Hq):
            a = np.array([qr[i, h] @ kk[h // 2, s] for s in range(hist + i + 1)]) / 8.0
            w = np.exp(a) / np.exp(a).sum()
            assert np.allclose(out[i, h], w @ vv[h // 2, :hist + i + 1], rtol=1e-12, atol=1e-12)


def test_a_tree_is_its_chains():
    """Each token's output is that of the chain of its ancestors alone."""
    n, Hq, Hkv, D, hist, L = 7, 2, 1, 64, 9, 20
    q, k, v = U.new_tokens("chains", 1, n, Hq, Hkv, D)
    parents = [-1, 0, 0, 1, -1, 2, 3]
    kc, vc = U.history("chains", 1, Hkv, L, D, [hist])
    tab = T.tables(L, D, U.THETA)
    for window, sinks in ((None, 0), (6, 2)):
        out, _ = T.attend(q[0], k[0], v[0], hist, parents, kc[0].copy(), vc[0].copy(), tab, window, sinks)
        for i, c in enumerate(T.kin(parents)):
            one, _ = T.attend(q[0, c], k[0, c], v[0, c], hist, T.chain(len(c)), kc[0].copy(), vc[0].copy(), tab, window, sinks)
            assert np.allclose(out[i], one[-1], rtol=1e-13, atol=0)


def test_accepting_a_path_leaves_the_cache_that_decoding_it_would():
    n, D, hist, L = 7, 64, 5, 16
    parents = [-1, 0, 0, 1, -1, 2, 3]
    q, k, v = U.new_tokens("path", 1, n, 2, 1, D)
    tab = T.tables(L, D, U.THETA)
    for leaf, c in enumerate(T.kin(parents)):
        kc, vc = U.history("path", 1, 1, L, D, [hist])
        k1, v1 = kc.copy(), vc.copy()
        T.attend(q[0], k[0], v[0], hist, parents, kc[0], vc[0], tab)
        assert T.accept(hist, parents, leaf, [kc[0], vc[0]]) == hist + len(c)
        T.attend(q[0, c], k[0, c], v[0, c], hist, T.chain(len(c)), k1[0], v1[0], tab)
        assert (kc[0, :, :hist + len(c)] == k1[0, :, :hist + len(c)]).all()
        assert (vc[0, :, :hist + len(c)] == v1[0, :, :hist + len(c)]).all()
    assert T.accept(hist, parents, -1, [kc[0], vc[0]]) == hist and T.accept(hist, parents, 7, [kc[0], vc[0]]) == hist


def test_null_arguments_are_refused(lib):
    from paper_2607_15865_gb300 import _lib
    nul, one = None, (ctypes.c_void_p * 1)()
    assert lib.attn_window_prefill_kv(nul, nul, nul, nul, 0, 4, 8, 0, nul, nul, nul, nul) == _lib.ATTN_EINVAL
    assert lib.attn_window_decode(nul, nul, nul, nul, nul, 1, 8, 0, nul, nul, nul, nul) == _lib.ATTN_EINVAL
    assert lib.attn_tree_decode(nul, nul, nul, nul, nul, nul, 1, 0, 0, nul, nul, nul, nul) == _lib.ATTN_EINVAL
    assert lib.attn_tree_accept(nul, nul, nul, nul, 1, one, one, 1, nul, nul) == _lib.ATTN_EINVAL


def test_a_window_past_any_int():
    from paper_2607_15865_gb300.attention import _int32
    assert [_int32(x) for x in (5, 2 ** 31, 2 ** 80, 0, -1, -2 ** 31 - 1, -2 ** 80)] == [5, 2 ** 31 - 1, 2 ** 31 - 1, 0, -1, -1, -1]
