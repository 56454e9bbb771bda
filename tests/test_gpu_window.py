"""window_prefill_kv against the float64 oracle, and against prefill_kv where the window hides nothing."""
import numpy as np
import pytest

from oracle import tree_oracle as T
from tests import tree_util as U

pytestmark = pytest.mark.gpu


def attention(B, Hq, Hkv, D, L):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, U.THETA)


def check(B, Hq, Hkv, D, hist, n, window, sinks, tag, kc=None, vc=None, new=None):
    attn = attention(B, Hq, Hkv, D, hist + n + 3)
    new = U.new_tokens(tag, B, n, Hq, Hkv, D) if new is None else new
    if kc is None:
        kc, vc = U.history(tag, B, Hkv, attn.max_len, D, [hist] * B)
    U.check(attn, new, [hist] * B, None, window, sinks, tag, kc=kc, vc=vc,
            call=lambda args, gk, gv, out: attn.window_prefill_kv(*args, hist, window, gk, gv, sinks=sinks, out=out))


# windows within a tile, of whole tiles, past everything; sinks that end in the first tile, at its border, in the window
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hist,n,window,sinks", [
    (0, 1, 1, 0), (0, 8, 3, 1), (0, 200, 1, 0), (0, 300, 64, 4), (100, 130, 128, 0), (129, 257, 127, 128), (128, 256, 129, 129),
    (600, 300, 200, 4), (600, 300, 200, 300), (1000, 64, 100, 0), (1000, 1, 300, 5), (1000, 65, 1100, 3), (777, 500, 5000, 0),
    (500, 140, 256, 257), (900, 129, 383, 385)])
def test_windows(D, hist, n, window, sinks):
    check(1, 4, 2, D, hist, n, window, sinks, f"pre{D}{hist}{n}{window}{sinks}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hq,Hkv,hist,n,window", [(2, 28, 4, 500, 77, 100), (3, 8, 8, 300, 20, 64), (1, 16, 1, 900, 40, 500),
                                                    (1, 40, 8, 1500, 16, 300), (4, 7, 1, 0, 150, 33), (2, 32, 8, 700, 300, 450)])
def test_heads_and_batches(D, B, Hq, Hkv, hist, n, window):
    check(B, Hq, Hkv, D, hist, n, window, 4, f"heads{D}{Hq}{n}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n", [9, 150])
def test_masked_places_reach_no_output(D, value, n):
    """NaN or infinities outside every window, past the last token and, with a few in places that some see, just in those."""
    hist, window, sinks = 400, 100, 5
    tag = f"masked{D}{n}"
    kc, vc = U.history(tag, 1, 2, hist + n + 3, D, [hist])
    x = T.f32_to_bf16(np.array([value], np.float32))[0]
    kc[:, :, 5:hist - window + 1] = x
    vc[:, :, 5:hist - window + 1] = x
    check(1, 8, 2, D, hist, n, window, sinks, tag + " outside", kc.copy(), vc.copy())
    vc[0, 1, hist - window + 3, 3] = x   # seen by the first three tokens alone
    vc[0, 0, 350, 11] = x                # by those before position 450
    new = U.new_tokens(tag, 1, n, 8, 2, D)
    new[2][0, n // 2, 1, 5] = x          # by the tokens from there on
    if value != value:
        new[1][0, n - 2, 0, 9] = x
    check(1, 8, 2, D, hist, n, window, sinks, tag + " inside", kc, vc, new)


@pytest.mark.parametrize("D,n,hist", [(128, 512, 1536), (64, 300, 700), (128, 20, 900)])
def test_a_window_that_hides_nothing(D, n, hist):
    """The same outputs as prefill_kv up to the order of float sums and a rounding of each weight and result."""
    import torch
    attn = attention(1, 8, 2, D, hist + n)
    tag = f"all{D}{n}"
    new = [U.dev(x) for x in U.new_tokens(tag, 1, n, 8, 2, D)]
    kc, vc = (U.dev(x) for x in U.history(tag, 1, 2, hist + n, D, [hist]))
    k2, v2 = kc.clone(), vc.clone()
    a = attn.prefill_kv(*new, hist, kc, vc)
    b = attn.window_prefill_kv(*new, hist, hist + n, k2, v2)
    assert torch.equal(kc.view(torch.int16), k2.view(torch.int16)) and torch.equal(vc.view(torch.int16), v2.view(torch.int16))
    # two roundings of a result (2^-8 each), and of the weights on both sides (2^-8 of a mass of at most the largest |v|)
    bar = 2 ** -8 * 2.1 * (a.float().abs() + vc.float().nan_to_num().abs().max())
    assert ((a.float() - b.float()).abs() <= bar).all()


def test_a_prompt_in_chunks():
    """A prompt cut into chunks gives what it gives whole, as far as each is exact."""
    Hq, Hkv, D, L, window, sinks = 8, 2, 128, 700, 150, 4
    attn = attention(1, Hq, Hkv, D, L)
    new = U.new_tokens("cut", 1, L, Hq, Hkv, D)
    kc, vc = U.history("cut", 1, Hkv, L, D, [0])
    ref, mass = U.want(new, [0], [T.chain(L)], kc, vc, L, window, sinks)
    gk, gv = (U.dev(np.full((1, Hkv, L, D), U.NAN)) for _ in "kv")
    at = 0
    for n in (300, 1, 37, 200, 162):
        out = attn.window_prefill_kv(*(U.dev(x[:, at:at + n]) for x in new), at, window, gk, gv, sinks=sinks)
        U.close(out, ref[:, at:at + n], mass[:, at:at + n], f"chunk at {at}")
        at += n
    assert (U.bits(gk) == kc).all() and (U.bits(gv) == vc).all() and attn.device_error() == 0


def test_graph_and_stream():
    import torch
    hist, n, window = 300, 140, 120
    attn = attention(1, 8, 2, 128, 500)
    new = U.new_tokens("wgraph", 1, n, 8, 2, 128)
    kc, vc = U.history("wgraph", 1, 2, 500, 128, [hist])
    gk, gv = U.dev(kc), U.dev(vc)
    args = [U.dev(x) for x in new]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = attn.window_prefill_kv(*args, hist, window, gk, gv, stream=side)
    side.synchronize()
    ref = U.want(new, [hist], [T.chain(n)], kc, vc, 500, window)
    U.close(out, *ref, "side stream")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        again = attn.window_prefill_kv(*args, hist, window, gk, gv)
    again.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, out)
