"""window_decode of one token, which runs on the decode kernel: how its splits meet (a cluster, global memory, several waves,
two CTAs per SM at head_dim 64), where the tiles of the sinks and of the window begin and end, what lies outside them."""
import numpy as np
import pytest

from oracle import tree_oracle as T
from tests import tree_util as U

pytestmark = pytest.mark.gpu
HIST_RANGE = 1


def attention(B, Hq, Hkv, D, L):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, U.THETA)


# few items (one wave, clusters), middling (global memory), more than the SMs (several waves); one to sixteen heads per kv head
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,L,window,sinks", [
    (1, 8, 8, 3000, 1500, 4), (2, 28, 4, 2500, 900, 130), (3, 16, 1, 4000, 3900, 0), (8, 32, 8, 1200, 700, 5),
    (24, 32, 8, 1500, 1000, 4), (40, 8, 4, 700, 64, 300), (5, 40, 8, 2000, 1, 0), (2, 4, 2, 1300, 5000, 5000)])
def test_batches(D, B, Hq, Hkv, L, window, sinks):
    r = np.random.default_rng([D, B, L])
    lens = [int(x) for x in r.integers(0, L, B)]
    lens[0], lens[-1] = L - 1, (0 if B > 1 else L - 1)
    tag = f"one{D}{B}{Hq}{window}"
    U.check(attention(B, Hq, Hkv, D, L), U.new_tokens(tag, B, 1, Hq, Hkv, D), lens, None, window, sinks, tag)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (127, 0), (128, 128), (129, 127), (130, 129), (256, 3), (500, 600)])
def test_borders(D, window, sinks):
    """Histories around those of whole tiles, in one batch."""
    lens = [0, 1, 126, 127, 128, 129, 255, 256, 257, 383, 384, 511, 639, 640, 641]
    tag = f"border{D}{window}{sinks}"
    attn = attention(len(lens), 4, 2, D, 700)
    U.check(attn, U.new_tokens(tag, len(lens), 1, 4, 2, D), lens, None, window, sinks, tag)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_masked_places_reach_no_output(D, value):
    """NaN and infinities in every slot that is not seen, and a few in some that are."""
    lens, L, window, sinks = [800, 400, 1023, 130], 1024, 200, 70
    tag = f"one masked{D}"
    kc, vc = U.history(tag, 4, 2, L, D, lens)
    x = T.f32_to_bf16(np.array([value], np.float32))[0]
    for b, h in enumerate(lens):
        kc[b, :, sinks:max(h - window + 1, sinks)] = x
        vc[b, :, sinks:max(h - window + 1, sinks)] = x
    attn = attention(4, 8, 2, D, L)
    new = U.new_tokens(tag, 4, 1, 8, 2, D)
    U.check(attn, new, lens, None, window, sinks, tag + " outside", kc=kc.copy(), vc=vc.copy())
    vc[0, 1, lens[0] - window + 1, 3] = x
    vc[1, 0, sinks - 1, 9] = x
    new[2][2, 0, 1, 5] = x
    U.check(attn, new, lens, None, window, sinks, tag + " inside", kc=kc, vc=vc)


@pytest.mark.parametrize("D", [64, 128])
def test_sequences_that_are_skipped(D):
    lens = [100, -1, 200, 199, 2 ** 31 - 1, 0, -2 ** 31]
    attn = attention(7, 8, 2, D, 200)
    U.check(attn, U.new_tokens("one skip", 7, 1, 8, 2, D), lens, None, 50, 3, f"one skipped {D}", expect_err=HIST_RANGE)


@pytest.mark.parametrize("D,B,L", [(128, 1, 2000), (64, 1, 2000), (128, 16, 900), (64, 40, 900)])
def test_a_window_that_hides_nothing(D, B, L):
    """The outputs of decode, up to the roundings of the weights and of the result on both sides: the tiles that a split
    takes, and so the order of sums, may be others."""
    import torch
    attn = attention(B, 16, 4, D, L)
    new = [U.dev(x) for x in U.new_tokens(f"plain{D}{B}", B, 1, 16, 4, D)]
    lens = [(b * 37 + L - 1) % L for b in range(B)]
    kc, vc = (U.dev(x) for x in U.history(f"plain{D}{B}", B, 4, L, D, lens))
    k2, v2 = kc.clone(), vc.clone()
    a = attn.decode(*new, U.dev_i32(lens), kc, vc)
    b = attn.window_decode(*new, U.dev_i32(lens), L, k2, v2)
    assert torch.equal(kc.view(torch.int16), k2.view(torch.int16)) and torch.equal(vc.view(torch.int16), v2.view(torch.int16))
    bar = 2 ** -8 * 2.1 * (a.float().abs() + vc.float().nan_to_num().abs().max())
    assert ((a.float() - b.float()).abs() <= bar).all()


def test_graph_streams_and_other_calls_between():
    """One graph of windowed and plain decodes of the same context, whose counters they share, replayed at other lengths."""
    import torch
    B, L, D = 3, 1500, 128
    attn = attention(B, 8, 2, D, L)
    kc, vc = U.history("between", B, 2, L, D, [L] * B)
    gk, gv = U.dev(kc), U.dev(vc)
    new = U.new_tokens("between", B, 1, 8, 2, D)
    args, lens, roots = [U.dev(x) for x in new], U.dev_i32([0] * B), U.dev_i32([[-1]] * B)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = attn.window_decode(*args, lens, 300, gk, gv, stream=side)
    side.synchronize()
    U.close(out, *U.want(new, [0] * B, [T.chain(1)] * B, kc, vc, L, 300), "side stream")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wide = attn.window_decode(*args, lens, 1000, gk, gv, sinks=4)
        tree = attn.tree_decode(*args, lens, roots, gk, gv)
        narrow = attn.window_decode(*args, lens, 30, gk, gv)
        plain = attn.decode(*args, lens, gk, gv)
    for hist in ([1499, 3, 700], [0, 1000, 128], [640, 641, 1400]):
        lens.copy_(U.dev_i32(hist))
        g.replay()
        torch.cuda.synchronize()
        for out, w, s in ((wide, 1000, 4), (narrow, 30, 0), (plain, None, 0), (tree, None, 0)):
            U.close(out, *U.want(new, hist, [T.chain(1)] * B, kc, vc, L, w, s), f"replayed {w}")
    assert (U.bits(gk) == kc).all() and (U.bits(gv) == vc).all() and attn.device_error() == 0
