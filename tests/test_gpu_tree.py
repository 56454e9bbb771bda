"""tree_decode and window_decode against the float64 oracle: types of trees, lengths, windows, head layouts, refusals."""
import numpy as np
import pytest

from oracle import tree_oracle as T
from tests import tree_util as U

pytestmark = pytest.mark.gpu

HIST_RANGE, TREE = 1, 4


def attention(B, Hq, Hkv, D, L):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, U.THETA)


# lengths that end before, at and after a tile's border, new tokens that span one, one token over nothing
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hist,n", [(0, 1), (0, 64), (1, 2), (100, 64), (127, 1), (128, 1), (120, 16), (257, 33), (1000, 7)])
def test_lengths(D, hist, n):
    attn = attention(1, 8, 2, D, hist + n + 5)
    tag = f"len{D}{hist}{n}"
    new = U.new_tokens(tag, 1, n, 8, 2, D)
    U.check(attn, new, [hist], [U.random_tree(hist + n, n, 4)], 0, 0, tag)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (16, 1), (28, 4), (40, 8)])
@pytest.mark.parametrize("n", [1, 5, 26, 64])
def test_heads(D, Hq, Hkv, n):
    attn = attention(2, Hq, Hkv, D, 400)
    tag = f"heads{D}{Hq}{n}"
    new = U.new_tokens(tag, 2, n, Hq, Hkv, D)
    U.check(attn, new, [300, 130], [U.random_tree(n + b, n, 5) for b in range(2)], 0, 0, tag)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hist,n,window,sinks", [
    (500, 1, 1, 0), (500, 1, 128, 0), (500, 1, 129, 4), (500, 1, 10000, 0), (500, 9, 3, 1), (500, 9, 200, 130),
    (130, 20, 5, 128), (5, 40, 7, 12), (0, 64, 3, 2), (300, 64, 64, 0), (1000, 3, 300, 300), (700, 2, 10, 699), (700, 2, 10, 5000)])
def test_windows(D, hist, n, window, sinks):
    tag = f"win{D}{hist}{n}{window}{sinks}"
    attn = attention(1, 8, 2, D, hist + n)
    new = U.new_tokens(tag, 1, n, 8, 2, D)
    U.check(attn, new, [hist], None, window, sinks, tag + " chain")
    U.check(attn, new, [hist], [U.random_tree(hist, n, 3)], window, sinks, tag + " tree")


TREES = {
    "star": [-1] + [0] * 20, "roots": [-1] * 21, "chain": T.chain(21), "two chains": [-1, -1] + list(range(19)),
    "absent in the middle": [-1, 0, -2, 1, -2, 3, 0, -2] + [6] * 13, "none": [-2] * 21, "absent first": [-2, -1] + [1] * 19,
}


@pytest.mark.parametrize("name", TREES)
@pytest.mark.parametrize("D", [64, 128])
def test_trees(name, D):
    attn = attention(1, 4, 2, D, 170)
    new = U.new_tokens(name, 1, 21, 4, 2, D)
    U.check(attn, new, [140], [TREES[name]], 0, 0, f"tree {name} {D}")
    U.check(attn, new, [140], [TREES[name]], 4, 1, f"tree {name} {D} window")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,window", [(1, 700), (12, 0), (40, 90)])
def test_batches_of_mixed_lengths(D, n, window):
    """Lengths from none to long, trees of other numbers of tokens."""
    lens = [0, 1, 2000, 128, 777, 64, 1999, 300]
    B, L = len(lens), 2100
    attn = attention(B, 16, 4, D, L)
    new = U.new_tokens(f"mix{D}{n}", B, n, 16, 4, D)
    parents = [U.random_tree(b, n, 4, gone=(b * 5) % n) for b in range(B)]
    U.check(attn, new, lens, parents, window, 3, f"mixed {D} {n}")


@pytest.mark.parametrize("D,Hq,Hkv,n,hist", [(128, 8, 1, 1, 9000), (128, 40, 8, 64, 5000), (64, 8, 1, 64, 7000), (64, 32, 8, 1, 9000)])
def test_long_histories(D, Hq, Hkv, n, hist):
    attn = attention(1, Hq, Hkv, D, hist + n)
    tag = f"long{D}{Hq}{n}"
    new = U.new_tokens(tag, 1, n, Hq, Hkv, D)
    U.check(attn, new, [hist], [U.random_tree(n, n, 7)], 0, 0, tag)
    U.check(attn, new, [hist], None, 3000, 4, tag + " window")


def test_many_sequences():
    """More sequences than one launch counts."""
    B, D, L = 1100, 64, 40
    attn = attention(B, 2, 1, D, L)
    new = U.new_tokens("many", B, 3, 2, 1, D)
    lens = [(b * 7) % 37 for b in range(B)]
    U.check(attn, new, lens, [[-1, 0, 0] if b % 3 else [-1, -1, 1] for b in range(B)], 0, 0, "many")


@pytest.mark.parametrize("D", [64, 128])
def test_sequences_that_are_skipped(D):
    """Lengths outside the cache and parents that are none: those sequences alone are left as they were."""
    B, n, L = 9, 4, 200
    attn = attention(B, 8, 2, D, L)
    new = U.new_tokens(f"skip{D}", B, n, 8, 2, D)
    good = [-1, 0, 0, 1]
    lens = [196, 197, -1, 100, 100, 100, 200, 197, 2 ** 31 - 1]
    parents = [good, good, good, [0, 0, 0, 0], [-1, 0, 2, 0], [-2, 0, -1, -1], [-2] * 4, [-1, 0, 0, -2], good]
    U.check(attn, new, lens, parents, 0, 0, "skipped", expect_err=HIST_RANGE | TREE)
    U.check(attn, new, [196, 196, 3, 4, 5, 6, 7, 8, 9], None, 50, 0, "none skipped")
    U.check(attn, new, [196, 197, 3, 4, 5, 6, -7, 8, 9], None, 50, 0, "chains skipped", expect_err=HIST_RANGE)
    bad = [[-1, 0, 0, p] for p in (3, 64, -3, -2 ** 31, 2 ** 31 - 1, 2, 2, 2, 2)]
    U.check(attn, new, [50] * B, bad, 0, 0, "bad parents", expect_err=TREE)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n,window", [(1, 40), (30, 40), (64, 200)])
def test_masked_places_reach_no_output(D, value, n, window):
    """Slots outside every window, of strangers in the tree and past the last token hold NaN or infinities; so do some k and
    v that a few tokens see, and reach just those."""
    hist, L = 333, 460
    tag = f"masked{D}{n}"
    attn = attention(1, 8, 2, D, L)
    new = U.new_tokens(tag, 1, n, 8, 2, D)
    parents = [U.random_tree(n, n, 3)]
    kc, vc = U.history(tag, 1, 2, L, D, [hist])
    x = T.f32_to_bf16(np.array([value], np.float32))[0]
    far = hist - window - 70
    kc[:, :, 5:hist - window + 1] = x  # slots 4 .. are before every window
    vc[:, :, 5:hist - window + 1] = x
    U.check(attn, new, [hist], parents, window, 5, tag + " outside", kc=kc.copy(), vc=vc.copy())
    vc[0, 1, hist - window + 2, 3] = x  # seen by the first tokens alone
    if n > 8:
        new[2][0, 5, 0, 7] = x  # seen by token 5 and its descendants
        new[1][0, 6, 1, 9] = np.uint16(0x7FC0)
    assert far < hist
    U.check(attn, new, [hist], parents, window, 5, tag + " inside", kc=kc, vc=vc)
    U.check(attn, new, [hist], None, window, 5, tag + " chain", kc=kc, vc=vc)


def test_large_values_keep_their_range():
    """v of 2^100 in masked and seen places, scores whose exponentials span the float range."""
    hist, n, D, L = 200, 6, 128, 256
    attn = attention(1, 8, 2, D, L)
    q, k, v = U.new_tokens("range", 1, n, 8, 2, D)
    q = T.f32_to_bf16(T.bf16_to_f64(q).astype(np.float32) * 12)
    kc, vc = U.history("range", 1, 2, L, D, [hist])
    vc[0, 0, 150:170] = 0x7180
    vc[0, 0, 0:20] = 0x7180
    U.check(attn, (q, k, v), [hist], [[-1, 0, 0, 1, 1, 2]], 40, 0, "range", kc=kc, vc=vc)


def test_refusals():
    import torch
    attn = attention(2, 8, 2, 128, 100)
    new = [U.dev(x) for x in U.new_tokens("no", 2, 3, 8, 2, 128)]
    kc, vc = (torch.zeros(2, 2, 100, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    lens, par = U.dev_i32([5, 6]), U.dev_i32([[-1, 0, 0]] * 2)
    from paper_2607_15865_gb300._lib import AttnError
    for bad in (0, -1, -2 ** 40):
        with pytest.raises(AttnError):
            attn.window_decode(*new, lens, bad, kc, vc)
        with pytest.raises(AttnError):
            attn.window_prefill_kv(*new, 0, bad, kc, vc)
    with pytest.raises(AttnError):
        attn.tree_decode(*new, lens, par, kc, vc, window=-1)
    for call in (lambda: attn.window_decode(*new, lens, 5, kc, vc, sinks=-1),
                 lambda: attn.window_prefill_kv(*new, 98, 5, kc, vc), lambda: attn.window_prefill_kv(*new, -1, 5, kc, vc),
                 lambda: attn.tree_decode(*new, lens, par, kc, vc, sinks=-1)):
        with pytest.raises(AttnError):
            call()
    many = [U.dev(x) for x in U.new_tokens("no", 2, 65, 8, 2, 128)]
    none = [x[:, :0].contiguous() for x in new]
    for x in (many, none):
        with pytest.raises(AttnError):
            attn.window_decode(*x, lens, 5, kc, vc)
        with pytest.raises(AttnError):
            attn.tree_decode(*x, lens, torch.full((2, x[0].shape[1]), -1, dtype=torch.int32, device="cuda"), kc, vc)
    for p in (par.long(), par[:1], par[:, :2], par.t().contiguous().t(), par.cpu(), None):
        with pytest.raises(TypeError):
            attn.tree_decode(*new, lens, p, kc, vc)
    with pytest.raises(TypeError):
        attn.tree_decode(*new, lens.long(), par, kc, vc)
    with pytest.raises(TypeError):
        attn.window_decode(new[0].float(), *new[1:], lens, 5, kc, vc)
    with pytest.raises(ValueError):
        attn.window_decode(new[0], new[1][:, :, :1].contiguous(), new[2], lens, 5, kc, vc)
    with pytest.raises(ValueError):
        attn.window_decode(*new, lens, 5, kc[:, :, :50].contiguous(), vc)
    assert not kc.any() and not vc.any() and attn.device_error() == 0


def test_graph_and_streams():
    """Captured once, replayed with new inputs, lengths and trees; a call on a stream of its own."""
    import torch
    B, n, D, L = 2, 9, 128, 600
    attn = attention(B, 8, 2, D, L)
    tag = "graph"
    steps = [(U.new_tokens(f"{tag}{i}", B, n, 8, 2, D), lens, [U.random_tree(10 * i + b, n, 4) for b in range(B)])
             for i, lens in enumerate(([500, 3], [100, 590], [256, 128]))]
    kc, vc = U.history(tag, B, 2, L, D, [L, L])
    gk, gv = U.dev(kc), U.dev(vc)
    new, lens, par = [U.dev(x) for x in steps[0][0]], U.dev_i32(steps[0][1]), U.dev_i32(steps[0][2])
    side = torch.cuda.Stream()
    out = attn.tree_decode(*new, lens, par, gk, gv, stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attn.tree_decode(*new, lens, par, gk, gv, out=out)
        win = attn.window_decode(*new, lens, 77, gk, gv, sinks=2)
    U.want(steps[0][0], steps[0][1], steps[0][2], kc, vc, L)
    for inputs, hist, parents in steps:
        for t, x in zip(new, inputs):
            t.copy_(U.dev(x))
        lens.copy_(U.dev_i32(hist))
        par.copy_(U.dev_i32(parents))
        g.replay()
        torch.cuda.synchronize()
        U.close(out, *U.want(inputs, hist, parents, kc, vc, L), "replayed tree")
        U.close(win, *U.want(inputs, hist, [T.chain(n)] * B, kc, vc, L, 77, 2), "replayed window")
        assert (U.bits(gk) == kc).all() and (U.bits(gv) == vc).all()
    assert attn.device_error() == 0
    side.wait_stream(torch.cuda.current_stream())
    out2 = attn.tree_decode(*new, lens, par, gk, gv, stream=side)
    side.synchronize()
    assert torch.equal(out2, out)


def test_calls_repeat_bit_for_bit():
    import torch
    attn = attention(3, 40, 8, 128, 5000)
    new = [U.dev(x) for x in U.new_tokens("repeat", 3, 20, 40, 8, 128)]
    kc, vc = (U.dev(x) for x in U.history("repeat", 3, 8, 5000, 128, [5000] * 3))
    lens, par = U.dev_i32([4900, 77, 2500]), U.dev_i32([U.random_tree(b, 20, 4) for b in range(3)])
    first = attn.tree_decode(*new, lens, par, kc, vc)
    for _ in range(5):
        assert torch.equal(attn.tree_decode(*new, lens, par, kc, vc), first)
