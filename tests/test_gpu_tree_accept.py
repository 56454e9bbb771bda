"""tree_accept against the oracle, and a run of drafts verified and accepted over several layers."""
import numpy as np
import pytest

from oracle import tree_oracle as T
from tests import tree_util as U

pytestmark = pytest.mark.gpu

HIST_RANGE, TREE = 1, 4


def attention(B, Hq, Hkv, D, L):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, U.THETA)


def check(attn, lens, parents, leaves, layers, tag, expect_err=0):
    B, H, L, D = attn._cache
    caches = [(U.bf16(tag, f"k{i}", (B, H, L, D)), U.bf16(tag, f"v{i}", (B, H, L, D))) for i in range(layers)]
    gpu = [(U.dev(k), U.dev(v)) for k, v in caches]
    got = attn.tree_accept(U.dev_i32(lens), U.dev_i32(parents), U.dev_i32(leaves), gpu)
    assert attn.device_error() == expect_err
    new = [T.accept(lens[b], parents[b], leaves[b], [x[b] for kv in caches for x in kv]) for b in range(B)]
    assert got.tolist() == new
    for (k, v), (gk, gv) in zip(caches, gpu):
        assert (U.bits(gk) == k).all() and (U.bits(gv) == v).all(), tag


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,width", [(1, 1), (2, 1), (8, 3), (33, 5), (64, 1), (64, 8), (64, 64)])
def test_every_leaf(D, n, width):
    """As many sequences as there are answers: each token of the tree, and none."""
    leaves = list(range(-1, n))
    B = len(leaves)
    attn = attention(B, 2, 2, D, 80)
    parents = [U.random_tree(b, n, width, roots=0.05) for b in range(B)]
    check(attn, [(5 * b) % 17 for b in range(B)], parents, leaves, 2, f"leaf{D}{n}{width}")


def test_paths_whose_slots_overlap():
    """Rows that move to slots that other rows leave."""
    attn = attention(4, 2, 1, 128, 40)
    parents = [[-1, -1] + list(range(1, 13)), [-1, -1, -1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12],
               [-2, -1] + list(range(1, 13)), T.chain(14)]
    check(attn, [3, 26, 0, 20], parents, [13] * 4, 1, "overlap")


@pytest.mark.parametrize("layers", [1, 40, 128, 129])
def test_layers(layers):
    attn = attention(2, 4, 2, 64, 50)
    check(attn, [10, 40], [U.random_tree(b, 10, 3) for b in range(2)], [9, 7], layers, f"layers{layers}")


def test_sequences_that_are_skipped():
    attn = attention(9, 4, 2, 128, 60)
    good = [-1, 0, 0, 1]
    lens = [56, 57, -1, 20, 20, 20, 20, 60, 57]
    parents = [good, good, good, [0] * 4, good, good, [-1, 0, -2, 1], [-2] * 4, [-1, 0, 0, -2]]
    leaves = [3, 3, 3, 3, 4, -2, 2, -1, 2]
    check(attn, lens, parents, leaves, 2, "skipped", expect_err=HIST_RANGE | TREE)


def test_refusals():
    import torch

    from paper_2607_15865_gb300._lib import AttnError
    attn = attention(2, 4, 2, 64, 50)
    cache = lambda: tuple(torch.ones(2, 2, 50, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv")  # noqa: E731
    lens, par, leaf = U.dev_i32([5, 6]), U.dev_i32([[-1, 0]] * 2), U.dev_i32([1, 0])
    kv = cache()
    with pytest.raises(AttnError):
        attn.tree_accept(lens, par, leaf, [])
    with pytest.raises(AttnError):
        attn.tree_accept(lens, par, leaf, [kv], new_len=lens)
    with pytest.raises(ValueError):
        attn.tree_accept(lens, par, leaf, [kv, kv])
    with pytest.raises(ValueError):
        attn.tree_accept(lens, par, leaf, [(kv[0], kv[0])])
    with pytest.raises(ValueError):
        attn.tree_accept(lens, par, leaf, [(kv[0], kv[1][:, :, :40].contiguous())])
    for bad in ((lens.long(), par, leaf), (lens, par.long(), leaf), (lens, par, leaf[:1]), (lens, par[0], leaf)):
        with pytest.raises(TypeError):
            attn.tree_accept(*bad, [kv])
    with pytest.raises(AttnError):
        attn.tree_accept(lens, torch.full((2, 65), -1, dtype=torch.int32, device="cuda"), leaf, [kv])
    overlap = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(AttnError):
        attn.tree_accept(overlap[:2], par, leaf, [kv], new_len=overlap[1:])
    torch.cuda.synchronize()
    assert all((x == 1).all() for x in kv) and attn.device_error() == 0


def test_a_run_of_drafts():
    """Prompt, then trees verified and accepted, then a token decoded, in two layers (one with a window), from one graph per
    tree size: the caches and outputs are those of the accepted tokens decoded one after the other."""
    import torch
    B, Hq, Hkv, D, L, P, n, W = 2, 8, 2, 128, 400, 150, 12, 100
    attn = attention(B, Hq, Hkv, D, L)
    kc, vc = (np.zeros((2, B, Hkv, L, D), np.uint16) for _ in "kv")  # per layer, on the host
    gpu = [(U.dev(kc[i]), U.dev(vc[i])) for i in range(2)]
    prompt = U.new_tokens("run prompt", B, P, Hq, Hkv, D)
    dev = [U.dev(x) for x in prompt]
    outs = [attn.prefill(*dev, *gpu[0]), attn.window_prefill_kv(*dev, 0, W, *gpu[1], sinks=4)]
    for i, (w, s) in enumerate(((None, 0), (W, 4))):
        U.close(outs[i], *U.want(prompt, [0] * B, [T.chain(P)] * B, kc[i], vc[i], L, w, s), f"prompt {i}")
    lens, next_len = U.dev_i32([P] * B), U.dev_i32([0] * B)
    leaf, par = U.dev_i32([0] * B), U.dev_i32([T.chain(n)] * B)
    new = [torch.empty_like(U.dev(x)) for x in U.new_tokens("run 0", B, n, Hq, Hkv, D)]
    res = [torch.zeros_like(new[0]) for _ in range(2)]

    def step():
        attn.tree_decode(*new, lens, par, *gpu[0], out=res[0])
        attn.tree_decode(*new, lens, par, *gpu[1], window=W, sinks=4, out=res[1])
        attn.tree_accept(lens, par, leaf, gpu, new_len=next_len)
        lens.copy_(next_len)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    hist = [P] * B
    for t in range(4):
        x = U.new_tokens(f"run {t}", B, n, Hq, Hkv, D)
        parents = [U.random_tree(100 * t + b, n, 3, gone=2 * b) for b in range(B)]
        leaves = [(5 * t + 4) % n, 9 - t]
        for a, c in zip(new, x):
            a.copy_(U.dev(c))
        par.copy_(U.dev_i32(parents))
        leaf.copy_(U.dev_i32(leaves))
        g.replay()
        torch.cuda.synchronize()
        rows = U.rows_written(hist, parents, L)
        for i, (w, s) in enumerate(((None, 0), (W, 4))):
            ref, mass = U.want(x, hist, parents, kc[i], vc[i], L, w, s)
            U.close(res[i], ref, mass, f"step {t} layer {i}", rows)
        after = [T.accept(hist[b], parents[b], leaves[b], [c[i][b] for c in (kc, vc) for i in range(2)]) for b in range(B)]
        hist = after
        assert lens.tolist() == hist
        for i in range(2):
            assert (U.bits(gpu[i][0]) == kc[i]).all() and (U.bits(gpu[i][1]) == vc[i]).all()
    one = U.new_tokens("run end", B, 1, Hq, Hkv, D)
    d = [U.dev(x) for x in one]
    U.close(attn.decode(*d, lens, *gpu[0]), *U.want(one, hist, [[-1]] * B, kc[0], vc[0], L), "decoded token")
    U.close(attn.window_decode(*d, lens, W, *gpu[1], sinks=4), *U.want(one, hist, [[-1]] * B, kc[1], vc[1], L, W, 4),
            "decoded token, window")
    assert attn.device_error() == 0


def test_new_lengths_over_an_input_are_refused():
    """Other blocks of the launch may still read what the first one has written."""
    import torch

    from paper_2607_15865_gb300._lib import AttnError
    attn = attention(2, 4, 2, 64, 50)
    kv = tuple(torch.ones(2, 2, 50, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    x = torch.zeros(12, dtype=torch.int32, device="cuda")
    lens, leaf, par = x[:2], x[4:6], x[8:12].view(2, 2).fill_(-1)
    for bad in (leaf, x[3:5], x[5:7], x[8:10], x[7:9], x[1:3]):
        with pytest.raises(AttnError):
            attn.tree_accept(lens, par, leaf, [kv], new_len=bad)
    assert attn.tree_accept(lens, par, leaf, [kv], new_len=x[2:4]).tolist() == [1, 1] and attn.device_error() == 0
    assert attn.tree_accept(lens, par, leaf, [kv], new_len=x[6:8]).tolist() == [1, 1]
