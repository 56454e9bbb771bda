"""tree_decode and window_prefill_kv where a CTA walks many pieces of work, and where their waits run out."""
import numpy as np
import pytest

from oracle import tree_oracle as T
from tests import tree_util as U

pytestmark = pytest.mark.gpu
TIMEOUT = 2


def attention(B, Hq, Hkv, D, L):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, U.THETA)


# many short items per CTA, among some that several share; one, two and three groups of rows, the last of them with one tile and two
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,n,window", [(60, 32, 8, 2, 0), (100, 16, 8, 9, 150), (20, 32, 8, 40, 0), (30, 40, 8, 64, 0),
                                               (12, 16, 1, 40, 400), (9, 64, 4, 24, 0), (33, 16, 16, 64, 90),
                                               (130, 10, 2, 60, 0)])
def test_many_segments(D, B, Hq, Hkv, n, window):
    r = np.random.default_rng([D, B, n])
    L = 1500
    lens = [int(x) for x in (r.random(B) ** 4 * (L - n))]
    lens[B // 2], lens[-1] = L - n, 0
    tag = f"many{D}{B}{n}"
    parents = [U.random_tree(b, n, 5, gone=b % n if b % 3 else 0) for b in range(B)]
    U.check(attention(B, Hq, Hkv, D, L), U.new_tokens(tag, B, n, Hq, Hkv, D), lens, parents, window, 3, tag)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [3, 30])
def test_values_that_are_not_finite_in_some_segments(D, n):
    """In every third sequence, where some rows alone see them: the others of the same CTA are as they would be."""
    B, L, W = 45, 700, 100
    r = np.random.default_rng([D, n])
    lens = [int(x) for x in r.integers(0, L - n, B)]
    tag = f"odd{D}{n}"
    kc, vc = U.history(tag, B, 8, L, D, lens)
    new = U.new_tokens(tag, B, n, 16, 8, D)
    for b in range(0, B, 3):
        vc[b, b % 8, max(lens[b] - W // 2, 0), 5] = 0x7F80
        new[2][b, n - 2, (b + 1) % 8, 7] = 0x7FC0
    U.check(attention(B, 16, 8, D, L), new, lens, [U.random_tree(b, n, 3) for b in range(B)], W, 2, tag, kc=kc, vc=vc)


@pytest.mark.parametrize("D,value", [(64, np.nan), (128, np.inf)])
def test_a_windowed_prompt_of_many_rounds(D, value):
    """More query tiles than SMs, with values that are not finite at a few places of some heads."""
    B, Hq, Hkv, hist, n, W = 5, 32, 8, 200, 600, 150
    tag = f"rounds{D}"
    attn = attention(B, Hq, Hkv, D, hist + n)
    kc, vc = U.history(tag, B, Hkv, hist + n, D, [hist] * B)
    new = U.new_tokens(tag, B, n, Hq, Hkv, D)
    x = T.f32_to_bf16(np.array([value], np.float32))[0]
    for b in range(B):
        vc[b, b, 150, 3] = x
        new[2][b, 100 + 90 * b, (b + 3) % Hkv, 11] = x
    U.check(attn, new, [hist] * B, None, W, 4, tag, kc=kc, vc=vc,
            call=lambda args, gk, gv, out: attn.window_prefill_kv(*args, hist, W, gk, gv, sinks=4, out=out))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,n,lens", [(1, 32, 8, 8, [900]), (1, 40, 8, 64, [900]), (20, 16, 8, 5, None), (3, 32, 8, 1, None)])
def test_waits_that_run_out(D, B, Hq, Hkv, n, lens):
    """With a limit of 1 ns each call returns and says so; after that the same context is right again."""
    L, W = 1000, 300
    lens = [(b * 311 + 60) % (L - 70) for b in range(B)] if lens is None else lens
    tag = f"wait{D}{B}{n}"
    attn = attention(B, Hq, Hkv, D, L)
    new = U.new_tokens(tag, B, n, Hq, Hkv, D)
    kc, vc = U.history(tag, B, Hkv, L, D, lens)
    parents = [U.random_tree(b, n, 4) for b in range(B)]
    args = [U.dev(x) for x in new]
    attn.set_wait_limit(1)
    try:
        for call in (lambda k, v: attn.tree_decode(*args, U.dev_i32(lens), U.dev_i32(parents), k, v),
                     lambda k, v: attn.window_decode(*args, U.dev_i32(lens), W, k, v, sinks=4),
                     lambda k, v: attn.window_prefill_kv(*args, min(lens), W, k, v, sinks=4)):
            call(U.dev(kc), U.dev(vc))
            assert attn.device_error() & TIMEOUT
    finally:
        attn.set_wait_limit(0)
    U.check(attn, new, lens, parents, 0, 0, tag + " tree after", kc=kc, vc=vc)
    U.check(attn, new, lens, None, W, 4, tag + " window after", kc=kc, vc=vc)


def test_two_contexts_at_once():
    """Calls of two contexts on two streams, whose CTAs wait for others of their own launch: the same as one after the other."""
    import torch
    runs = []
    for i, (Hq, Hkv, n, hist) in enumerate(((32, 8, 8, 2900), (40, 8, 30, 1500))):
        attn = attention(1, Hq, Hkv, 128, 3000)
        args = [U.dev(x) for x in U.new_tokens(f"two{i}", 1, n, Hq, Hkv, 128)]
        kc, vc = (U.dev(x) for x in U.history(f"two{i}", 1, Hkv, 3000, 128, [hist]))
        lens, par = U.dev_i32([hist]), U.dev_i32([U.random_tree(i, n, 4)])
        runs.append((attn, lambda out=None, s=None, a=attn, x=(*args, lens, par, kc, vc): a.tree_decode(*x, out=out, stream=s)))
    alone = [call() for _, call in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    outs = [[torch.zeros_like(x) for _ in range(10)] for x in alone]
    torch.cuda.synchronize()
    for k in range(10):
        for (_, call), s, out in zip(runs, streams, outs):
            call(out[k], s)
    torch.cuda.synchronize()
    for (attn, _), ref, out in zip(runs, alone, outs):
        assert attn.device_error() == 0 and all(torch.equal(x, ref) for x in out)
