"""The 4-bit cache on the GPU: append, read, decode and prefill_kv against 64 bits (bars: kv4_util)."""
import numpy as np
import pytest

from oracle import kv4_oracle as K
from tests import kv4_util as U

pytestmark = pytest.mark.gpu

DEV_ERR_HIST = 1


def context(B, Hq, Hkv, D, L, theta=1.0e6):
    from paper_2607_15865_gb300.attention import Attention
    return Attention(B, Hq, Hkv, D, L, theta)


def slots(L):
    return (L + 63) // 64 * 64


def run_append(attn, cache, ref, tag, hist, n, k=None, v=None):
    """Append n tokens on the device and in ref (a K.Cache, updated)."""
    B, Hkv, D = attn.batch, attn.n_kv_heads, attn.head_dim
    _, k0, v0 = U.new_tokens(tag, B, n, Hkv, Hkv, D)
    k, v = k0 if k is None else k, v0 if v is None else v
    attn.kv4_append(U.dev_bf16(k), U.dev_bf16(v), hist, cache)
    tab = K.tables(attn.max_len, D, attn.rope_theta)
    pos = np.arange(hist, hist + n)
    for b in range(B):
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])


# ------------------------------------------------------------------ append and read

@pytest.mark.parametrize("B,Hkv,D,L,hist,n", [
    (1, 1, 64, 1, 0, 1),         # one slot
    (1, 2, 64, 32, 16, 8),
    (2, 3, 128, 100, 37, 63),    # up to the last slot, odd
    (1, 8, 128, 2048, 0, 777),
    (5, 1, 64, 129, 1, 127),
    (3, 4, 128, 65, 64, 1),
])
def test_append_is_bit_exact_and_leaves_other_slots(B, Hkv, D, L, hist, n):
    attn = context(B, Hkv, Hkv, D, L)
    ref = U.history(f"app{B}{Hkv}{D}", B, Hkv, slots(L), D, [hist] * B)
    cache = U.to_dev(ref, L)
    run_append(attn, cache, ref, f"app{B}{Hkv}{D}", hist, n)
    U.same_cache(cache, ref, "append")
    assert attn.device_error() == 0


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_special_values(D):
    """Zeros, one-signed groups, infinities, NaN, subnormal and very large values, in v (k keeps its bits
    at position 0, where RoPE is the identity)."""
    n, Hkv, L = 12, 2, 16
    v = U.bf16("special", "v", (1, n, Hkv, D))
    f = K.bf16_to_f64(v)
    f[0, 0] = 0.0
    f[0, 1] = np.abs(f[0, 1])
    f[0, 2] = -np.abs(f[0, 2])
    f[0, 3, 0, 5], f[0, 3, 1, 40] = np.inf, -np.inf
    f[0, 4, 0, 33] = np.nan
    f[0, 5] *= 2.0 ** -130
    f[0, 6] *= 2.0 ** 120
    f[0, 7] = 0.0
    f[0, 7, :, 1::32] = 15.0
    f[0, 8] = -0.0
    f[0, 9] *= 2.0 ** -40
    f[0, 9, 0, 3] = 7.5
    f[0, 10] = 3.0
    f[0, 11, :, ::2] = 1e-40
    v = K.f32_to_bf16(f)
    for t in range(n):
        attn = context(1, Hkv, Hkv, D, L)
        ref = K.Cache(1, Hkv, slots(L), D)
        cache = U.to_dev(ref, L)
        run_append(attn, cache, ref, "special", 0, 1, v[:, t:t + 1], v[:, t:t + 1])
        U.same_cache(cache, ref, f"token {t}")
        k, w = attn.kv4_read(cache, 0, 1)
        for t2, got in enumerate((k, w)):
            want = K.values(ref.codes[t2][:, :, :1], ref.scales[t2][:, :, :1])
            got = K.bf16_to_f64(U.host_bits(got))
            assert ((got == want) | (np.isnan(got) & np.isnan(want))).all(), f"token {t}"


@pytest.mark.parametrize("D", [64, 128])
def test_append_of_ranges_that_float_rounds_off(D):
    """Groups whose range is 15 times a scale but for a far smaller value of the other sign, either way round."""
    n, Hkv, L = 40, 1, 64
    r = np.random.default_rng(5)
    f = r.uniform(-0.2, 0.2, (1, n, Hkv, D // 32, 32))
    big = 15.0 * r.integers(8, 16, (1, n, Hkv, D // 32)) * 2.0 ** r.integers(-6, 3, (1, n, Hkv, D // 32))
    f *= big[..., None]
    f[..., 1::2] = np.abs(f[..., 1::2])
    for i in range(n):  # all of one sign, then one value of the other far below it (or none)
        sign = 1.0 if i % 2 else -1.0
        f[0, i] = sign * np.abs(f[0, i])
        f[0, i, :, :, 7] = sign * big[0, i]
        f[0, i, :, :, 9] = -sign * big[0, i] * 2.0 ** -(20 + i) * (i % 5 > 0)
    v = K.f32_to_bf16(f.reshape(1, n, Hkv, D))
    attn = context(1, Hkv, Hkv, D, L)
    ref = K.Cache(1, Hkv, slots(L), D)
    cache = U.to_dev(ref, L)
    run_append(attn, cache, ref, f"round{D}", 0, n, None, v)
    U.same_cache(cache, ref, "append")


@pytest.mark.parametrize("B,Hkv,D,L,first,count", [
    (1, 1, 64, 1, 0, 1), (2, 3, 128, 100, 37, 63), (1, 8, 128, 2048, 0, 2048), (3, 2, 64, 130, 129, 1),
    (2, 2, 128, 65, 3, 0),
])
def test_read_gives_the_values(B, Hkv, D, L, first, count):
    import torch
    attn = context(B, Hkv, Hkv, D, L)
    ref = U.history(f"read{D}", B, Hkv, slots(L), D, [L - L // 3] * B)  # NaN groups in the last third
    cache = U.to_dev(ref, L)
    got = attn.kv4_read(cache, first, count)
    for t in range(2):
        want = K.values(ref.codes[t][:, :, first:first + count], ref.scales[t][:, :, first:first + count])
        g = K.bf16_to_f64(U.host_bits(got[t]))
        assert g.shape == want.shape and ((g == want) | (np.isnan(g) & np.isnan(want))).all()
    assert len(attn.kv4_read(cache)) == 2 and attn.kv4_read(cache)[0].shape == (B, Hkv, L, D)
    U.same_cache(cache, ref, "read")
    torch.cuda.synchronize()


# ------------------------------------------------------------------ decode

def run_decode(attn, ref, tag, hist, n, kv=None, what="decode"):
    """One decode of n tokens per sequence at the lengths hist; compares outputs and cache; returns out."""
    import torch
    B, Hq, Hkv, D, L = attn.batch, attn.n_q_heads, attn.n_kv_heads, attn.head_dim, attn.max_len
    q, k, v = U.new_tokens(tag, B, n, Hq, Hkv, D)
    if kv is not None:
        kv(k, v)
    cache = U.to_dev(ref, L)
    out = torch.full((B, n, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lens = torch.tensor(hist, dtype=torch.int32, device="cuda")
    attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), lens, cache, out=out)
    tab = K.tables(L, D, attn.rope_theta)
    want, mass = np.full(out.shape, 7.0), np.full(out.shape, 7.0)
    bad = False
    for b, h in enumerate(hist):
        if h < 0 or h + n > L:
            bad = True
            continue
        pos = np.arange(h, h + n)
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
        want[b], mass[b] = K.attend(K.rope(q[b], pos, tab), pos, ref, b)
    torch.cuda.synchronize()
    assert attn.device_error() == (DEV_ERR_HIST if bad else 0)
    U.close(out, want, mass, what)
    U.same_cache(cache, ref, what)
    return out


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (5, 1), (14, 2), (16, 1), (32, 8), (8, 8)])
def test_decode_group_sizes(D, Hq, Hkv):
    attn = context(2, Hq, Hkv, D, 300)
    hist = [213, 64]
    run_decode(attn, U.history(f"dg{D}", 2, Hkv, slots(300), D, hist), f"dg{Hq}{Hkv}{D}", hist, 1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hist", [[0], [1], [31], [32], [33], [63, 64, 65], [127, 128, 129, 0], [998, 0, 999, 500, 1],
                                  [7] * 40])
def test_decode_lengths(D, hist):
    B = len(hist)
    attn = context(B, 8, 2, D, 1000)
    run_decode(attn, U.history(f"dl{D}", B, 2, slots(1000), D, hist), f"dl{D}", hist, 1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 5])
@pytest.mark.parametrize("hist", [
    [200] * 20,                                              # one item to a CTA, some without any
    [90] * 130,                                              # several
    [(37 * i) % 290 for i in range(40)],                     # mixed
    [-1, 5, 700, 900] + [60] * 20 + [900, 0, -7],            # with skipped ones, at either end
    [(53 * i) % 600 if i % 5 else 999 for i in range(150)],
    [-1] * 20,
])
def test_decode_whole_items_for_a_cta(D, n, hist):
    """Batches whose items go whole to the CTAs, several to one, and such as are cut."""
    attn = context(len(hist), 8, 4, D, 620)
    run_decode(attn, U.history(f"wi{D}", len(hist), 4, slots(620), D, [min(max(h, 0), 620) for h in hist]), f"wi{D}", hist, n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", [(4, 2, 2), (8, 2, 5), (8, 1, 16), (16, 1, 16), (5, 1, 3), (7, 7, 4), (8, 4, 8),
                                      (14, 2, 11)])
def test_decode_several_tokens(D, Hq, Hkv, n):
    hist = [150, 0, 31, 96 - n]
    attn = context(4, Hq, Hkv, D, 200)
    run_decode(attn, U.history(f"dm{D}", 4, Hkv, slots(200), D, hist), f"dm{Hq}{Hkv}{n}{D}", hist, n)


@pytest.mark.parametrize("B,Hq,Hkv,D,L,hist,n", [
    (1, 8, 2, 128, 8192, [8191], 1), (1, 40, 8, 128, 6000, [5999], 1), (2, 8, 1, 64, 9000, [8999, 4444], 1),
    (1, 8, 2, 128, 5000, [4990], 7), (9, 4, 2, 128, 4000, [3999, 17, 2048, 0, 1000, 3500, 33, 64, 1], 1),
])
def test_decode_long(B, Hq, Hkv, D, L, hist, n):
    attn = context(B, Hq, Hkv, D, L)
    run_decode(attn, U.history(f"long{B}{D}", B, Hkv, slots(L), D, hist), f"long{B}{D}", hist, n)


def ramp(B, top):
    """Lengths 0 .. top, the long ones not all at one end."""
    return [top * ((i * 7) % B) // (B - 1) for i in range(B)]


@pytest.mark.parametrize("B,Hq,Hkv,D,L,hist,n", [
    # few items, cut into pieces in proportion to the lengths
    (6, 8, 2, 128, 1500, ramp(6, 1499), 1), (31, 2, 1, 64, 900, ramp(31, 890), 3), (1, 64, 64, 128, 200, [150], 1),
    # more items than half the SMs: equal runs, which begin and end inside items
    (12, 16, 8, 128, 1300, ramp(12, 1299), 1), (12, 16, 8, 64, 2500, ramp(12, 2400), 1),
    (12, 16, 8, 128, 700, ramp(12, 690), 8), (20, 32, 8, 64, 600, ramp(20, 590), 4),
    (40, 4, 4, 128, 400, [399 - i for i in range(40)], 1), (5, 16, 16, 64, 4000, [3999, 0, 31, 3000, 64], 1),
    (90, 2, 1, 128, 100, ramp(90, 99), 1),
    # several launches
    (130, 2, 1, 64, 150, ramp(130, 149), 1), (129, 2, 2, 128, 70, ramp(129, 66), 2),
    # column groups of one kv head
    (3, 16, 1, 128, 300, [250, 0, 100], 5), (7, 32, 4, 64, 200, ramp(7, 180), 16),
])
def test_decode_cuts(B, Hq, Hkv, D, L, hist, n):
    attn = context(B, Hq, Hkv, D, L)
    run_decode(attn, U.history(f"cut{B}{Hkv}{D}", B, Hkv, slots(L), D, hist), f"cut{B}{Hq}{D}{n}", hist, n)


@pytest.mark.parametrize("B,Hkv", [(3, 2), (11, 8)])
def test_decode_with_nothing_to_do(B, Hkv):
    """Every length outside the cache: all skipped and flagged."""
    attn = context(B, 2 * Hkv, Hkv, 128, 64)
    hist = [64] * B
    out = run_decode(attn, U.history("none", B, Hkv, 64, 128, hist), "none", hist, 1)
    assert (out == 7).all()


def test_decode_leaves_its_counters_for_the_next_call():
    """Shared items merged again and again, by calls of several shapes and with attn_decode between them."""
    import torch
    attn = context(2, 8, 2, 128, 3000)
    hist = [2999, 1700]
    ref = U.history("again", 2, 2, slots(3000), 128, hist)
    kc = torch.zeros(2, 2, 3000, 128, dtype=torch.bfloat16, device="cuda")
    q, k, v = (U.dev_bf16(x) for x in U.new_tokens("again", 2, 1, 8, 2, 128))
    lens = torch.tensor([100, 2000], dtype=torch.int32, device="cuda")
    for i in range(3):
        run_decode(attn, U.copy(ref), f"again{i}", [h - i for h in hist], 1 + i)
        attn.decode(q, k, v, lens, kc, kc.clone())


def test_decode_in_a_graph():
    import torch
    attn = context(1, 8, 2, 128, 600)
    ref = U.history("graph", 1, 2, slots(600), 128, [500])
    cache = U.to_dev(ref, 600)
    q, k, v = U.new_tokens("graph", 1, 1, 8, 2, 128)
    dq, dk, dv = (U.dev_bf16(x) for x in (q, k, v))
    lens = torch.tensor([500], dtype=torch.int32, device="cuda")
    out = torch.empty_like(dq)
    attn.kv4_decode(dq, dk, dv, lens, cache, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attn.kv4_decode(dq, dk, dv, lens, cache, out=out)
    tab = K.tables(600, 128, attn.rope_theta)
    for step in range(3):
        out.zero_()
        lens.fill_(500 + step)
        g.replay()
        torch.cuda.synchronize()
        pos = np.array([500 + step])
        ref.write(0, pos, K.rope(k[0], pos, tab), v[0])
        U.close(out[0], *K.attend(K.rope(q[0], pos, tab), pos, ref, 0), f"replay {step}")
    U.same_cache(cache, ref, "graph")


def test_decode_wait_that_runs_out():
    """With a limit of 1 ns the wait for the new tokens' rows may run out: the call returns and says so at most, and
    the next one, with the default limit, is right."""
    attn = context(1, 8, 2, 128, 300)
    ref = U.history("limit", 1, 2, slots(300), 128, [250])
    import torch
    q, k, v = (U.dev_bf16(x) for x in U.new_tokens("limit", 1, 16, 8, 2, 128))
    lens = torch.tensor([250], dtype=torch.int32, device="cuda")
    attn.set_wait_limit(1)
    attn.kv4_decode(q, k, v, lens, U.to_dev(ref, 300))
    assert attn.device_error() in (0, 2)
    attn.set_wait_limit(0)
    run_decode(attn, ref, "limit", [250], 16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 3])
def test_decode_skips_and_flags_lengths_outside(D, n):
    hist = [10, -1, 65 - n, 66 - n, 2 ** 31 - 1, -2 ** 31, 0]
    attn = context(7, 4, 2, D, 65)
    ref = U.history(f"skip{D}", 7, 2, slots(65), D, [min(max(h, 0), 65) for h in hist])
    out = run_decode(attn, ref, f"skip{D}", hist, n)
    assert (out[1] == 7).all() and (out[3] == 7).all() and (out[5] == 7).all()


@pytest.mark.parametrize("D", [64, 128])
def test_decode_of_sharp_and_far_scores(D):
    """Scores of hundreds, rising and falling along the history: the running maximum moves often."""
    hist = [700]
    attn = context(1, 4, 1, D, 800)
    ref = U.history(f"sharp{D}", 1, 1, slots(800), D, hist)
    c, s = K.quantise(K.f32_to_bf16(K.values(ref.codes[0][:, :, :700], ref.scales[0][:, :, :700])
                                    * np.linspace(0.1, 30, 700)[None, None, :, None]))
    ref.codes[0][:, :, :700], ref.scales[0][:, :, :700] = K.pack(c), s
    run_decode(attn, ref, f"sharp{D}", hist, 2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k_exp,v_exp", [(0, 40), (0, -40), (-20, 0), (3, 60), (-45, -30)])
def test_decode_of_large_and_small_values(D, k_exp, v_exp):
    """Keys and values 2^k_exp and 2^v_exp times as large as the others'."""
    hist = [100]
    attn = context(1, 4, 2, D, 200)
    ref = U.history(f"mag{D}", 1, 2, slots(200), D, hist)
    for t, e in enumerate((k_exp, v_exp)):
        c, s = K.quantise(K.f32_to_bf16(K.values(ref.codes[t][:, :, :100], ref.scales[t][:, :, :100]) * 2.0 ** e))
        ref.codes[t][:, :, :100], ref.scales[t][:, :, :100] = K.pack(c), s
    def scaled(k, v):
        k[:] = K.f32_to_bf16(K.bf16_to_f64(k) * 2.0 ** k_exp)
        v[:] = K.f32_to_bf16(K.bf16_to_f64(v) * 2.0 ** v_exp)
    run_decode(attn, ref, f"mag{D}", hist, 2, scaled)


@pytest.mark.parametrize("D", [64, 128])
def test_decode_nan_in_the_history(D):
    """A NaN group of a key makes the heads that read it NaN; one of a value its 32 outputs."""
    hist = [300, 300]
    attn = context(2, 4, 2, D, 400)
    ref = U.history(f"nan{D}", 2, 2, slots(400), D, hist)
    ref.scales[0][0, 1, 17, 1] = K.NAN_SCALE
    ref.scales[1][1, 0, 299, D // 32 - 1] = K.NAN_SCALE
    out = run_decode(attn, ref, f"nan{D}", hist, 1)
    assert out[0, 0, 2:].isnan().all() and not out[0, 0, :2].isnan().any()
    assert out[1, 0, :2, D - 32:].isnan().all() and not out[1, 0, :, :D - 32].isnan().any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv,hist", [
    (2, [400, 300]),
    (2, [5000, 700]),      # parts of several CTAs
    (64, [400, 1500, 5]),  # runs over items
])
@pytest.mark.parametrize("n", [1, 9])
def test_decode_nan_in_many_neighbouring_keys(D, Hkv, hist, n):
    """Stretches of the history in which every key is NaN, one that a whole part consists of among them."""
    L, B = max(hist) + 20, len(hist)
    attn = context(B, 2 * Hkv, Hkv, D, L)
    ref = U.history(f"nans{D}", B, Hkv, slots(L), D, hist)
    ref.scales[0][0, 0, 64:128] = K.NAN_SCALE
    ref.scales[0][0, Hkv - 1, :hist[0] // 2] = K.NAN_SCALE
    out = run_decode(attn, ref, f"nans{D}", hist, n)
    assert out[0, :, :2].isnan().all() and out[0, :, -2:].isnan().all() and not out[1:].isnan().any()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv,hist", [(1, 100), (1, 5000), (80, 700)])
def test_decode_nan_of_a_value_whose_weight_is_next_to_nothing(D, Hkv, hist):
    """A NaN v is seen whatever its weight: the new key is so near to the first head's q that all others weigh less
    than 2^-150 there (what they add to the other values is less than a float holds, and is not compared)."""
    import torch
    attn = context(1, 2 * Hkv, Hkv, D, hist + 1)
    tag = f"faint{D}"
    ref = U.history(tag, 1, Hkv, slots(hist + 1), D, [hist])
    ref.scales[1][0, :, 3, 0] = K.NAN_SCALE
    q, k, v = U.new_tokens(tag, 1, 1, 2 * Hkv, Hkv, D)
    k = K.f32_to_bf16(20.0 * K.bf16_to_f64(q)[:, :, ::2])
    lens = torch.tensor([hist], dtype=torch.int32, device="cuda")
    out = attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), lens, U.to_dev(ref, hist + 1))
    assert out[..., :32].isnan().all() and not out[..., 32:].isnan().any()
    assert attn.device_error() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,n", [(2, 4), (8, 5)])
def test_decode_nan_in_a_new_token_reaches_only_later_ones(D, Hq, n):
    """Token 2's infinite k and NaN v are seen by tokens 2 .. n - 1 and not by 0 and 1."""
    hist = [61]
    attn = context(1, Hq, 2, D, 100)
    def odd(k, v):
        k[0, 2, 0, 5] = 0x7F80
        v[0, 2, 1, 33] = 0x7FC0
    out = run_decode(attn, U.history(f"late{D}", 1, 2, slots(100), D, hist), f"late{D}", hist, n, odd)
    assert not out[0, :2].isnan().any() and out[0, 2:, :Hq // 2].isnan().all()
    assert out[0, 2:, Hq // 2:, 32:64].isnan().all() and not out[0, 2:, Hq // 2:, :32].isnan().any()


# ------------------------------------------------------------------ prefill

def run_prefill(attn, cache, ref, tag, hist, n, workspace=None, what="prefill"):
    B, Hq, Hkv, D, L = attn.batch, attn.n_q_heads, attn.n_kv_heads, attn.head_dim, attn.max_len
    q, k, v = U.new_tokens(tag, B, n, Hq, Hkv, D)
    out = attn.kv4_prefill_kv(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), hist, cache, workspace)
    tab, pos = K.tables(L, D, attn.rope_theta), np.arange(hist, hist + n)
    want, mass = np.zeros(out.shape), np.zeros(out.shape)
    for b in range(B):
        ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
        want[b], mass[b] = K.attend(K.rope(q[b], pos, tab), pos, ref, b)
    U.close(out, want, mass, what)
    U.same_cache(cache, ref, what)
    assert attn.device_error() == 0
    return out


@pytest.mark.parametrize("B,Hq,Hkv,D,L,hist,n", [
    (1, 4, 2, 64, 32, 0, 16), (1, 4, 2, 64, 32, 16, 8), (1, 1, 1, 128, 1, 0, 1), (2, 14, 2, 128, 300, 77, 130),
    (1, 16, 1, 64, 700, 500, 77), (3, 5, 5, 128, 260, 1, 259), (1, 28, 4, 128, 512, 0, 300),
    # short chunks, through the decode and (33 columns, and 32 over a short history) the workspace
    (2, 8, 2, 128, 2200, 2100, 4), (2, 8, 2, 128, 2200, 2100, 8), (1, 6, 2, 64, 2200, 2150, 11), (1, 8, 2, 128, 300, 280, 8),
    (3, 4, 1, 64, 64, 0, 4), (12, 8, 8, 128, 100, 99, 1),
])
def test_prefill(B, Hq, Hkv, D, L, hist, n):
    attn = context(B, Hq, Hkv, D, L)
    ref = U.history(f"pre{B}{D}", B, Hkv, slots(L), D, [hist] * B)
    run_prefill(attn, U.to_dev(ref, L), ref, f"pre{B}{Hq}{D}", hist, n)


@pytest.mark.parametrize("Hq,Hkv,D,n", [(8, 2, 128, 12), (10, 2, 64, 9), (8, 2, 128, 13)])
def test_prefill_of_up_to_48_columns_over_a_long_history(Hq, Hkv, D, n):
    """Through the decode, and (52 columns) the workspace."""
    attn = context(1, Hq, Hkv, D, 8200)
    ref = U.history(f"pl{D}", 1, Hkv, slots(8200), D, [8100])
    run_prefill(attn, U.to_dev(ref, 8200), ref, f"pl{D}{n}", 8100, n)


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_nan_in_the_history(D):
    """Stretches of NaN keys, and a NaN group of a value."""
    attn = context(1, 4, 4, D, 800)
    ref = U.history(f"prenan{D}", 1, 4, slots(800), D, [600])
    ref.scales[0][0, 0, :400] = K.NAN_SCALE
    ref.scales[0][0, 1, 128:256] = K.NAN_SCALE
    ref.scales[1][0, 2, 77, 1] = K.NAN_SCALE
    out = run_prefill(attn, U.to_dev(ref, 800), ref, f"prenan{D}", 600, 150)
    assert out[0, :, :2].isnan().all() and out[0, :, 2, 32:64].isnan().all() and not out[0, :, 3].isnan().any()


def test_a_prompt_in_chunks_then_decodes_equals_its_cache():
    """Two chunks in one workspace, single and several tokens: each step is the stage over the cache so far."""
    import torch
    attn = context(2, 8, 2, 128, 256)
    ref = K.Cache(2, 2, slots(256), 128)
    cache = attn.kv4_cache()
    ws = torch.empty(attn.kv4_workspace(200), dtype=torch.uint8, device="cuda")
    run_prefill(attn, cache, ref, "chain0", 0, 150, ws, "first chunk")
    run_prefill(attn, cache, ref, "chain1", 150, 37, ws, "second chunk")
    tab = K.tables(256, 128, attn.rope_theta)
    for t, n in ((187, 1), (188, 3), (191, 1)):
        q, k, v = U.new_tokens(f"chain{t}", 2, n, 8, 2, 128)
        lens = torch.full((2,), t, dtype=torch.int32, device="cuda")
        out = attn.kv4_decode(U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v), lens, cache)
        pos = np.arange(t, t + n)
        for b in range(2):
            ref.write(b, pos, K.rope(k[b], pos, tab), v[b])
            U.close(out[b], *K.attend(K.rope(q[b], pos, tab), pos, ref, b), f"step {t}")
    U.same_cache(cache, ref, "chain")


def test_the_cache_is_the_bf16_cache_quantised():
    """kv4_append writes what quantising attn_prefill's bf16 cache gives."""
    import torch
    attn = context(1, 8, 4, 128, 200, 5.0e5)
    q, k, v = (U.dev_bf16(x) for x in U.new_tokens("bf16", 1, 200, 8, 4, 128))
    kc, vc = (torch.zeros(1, 4, 200, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    attn.prefill(q, k, v, kc, vc)
    cache = attn.kv4_cache()
    attn.kv4_append(k, v, 0, cache)
    for t, (x, codes, scales) in enumerate(((kc, cache.k_codes, cache.k_scales), (vc, cache.v_codes, cache.v_scales))):
        c, s = K.quantise(U.host_bits(x))
        assert (codes[:, :, :200].cpu().numpy() == K.pack(c)).all(), "kv"[t]
        assert (scales[:, :, :200].cpu().numpy().view(np.uint16) == s).all(), "kv"[t]


def test_memory_that_a_call_allocates_belongs_to_its_stream():
    """A workspace and outputs allocated by calls on another stream are not memory that the current stream still
    writes to."""
    import torch
    attn = context(1, 8, 2, 128, 1000)
    ref = U.history("pool", 1, 2, slots(1000), 128, [500])
    q, k, v = U.new_tokens("pool", 1, 300, 8, 2, 128)
    dq, dk, dv = U.dev_bf16(q), U.dev_bf16(k), U.dev_bf16(v)
    a, b = U.to_dev(ref, 1000), U.to_dev(ref, 1000)
    want = attn.kv4_prefill_kv(dq, dk, dv, 500, a)
    want_k, want_v = attn.kv4_read(a)
    sizes = [attn.kv4_workspace(800), want.nbytes, want_k.nbytes, want_v.nbytes]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    for cycles in (1, 200_000_000):  # 0.1 s, and then the writes (once before, to have the kernels loaded)
        torch.cuda._sleep(cycles)
        for x in blocks:
            x.fill_(0x7F)
    del blocks, x
    out = attn.kv4_prefill_kv(dq, dk, dv, 500, b, stream=st)
    got_k, got_v = attn.kv4_read(b, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(got_k[:, :, :800], want_k[:, :, :800])
    assert torch.equal(got_v[:, :, :800], want_v[:, :, :800])


def test_calls_on_another_stream():
    import torch
    attn = context(1, 8, 2, 128, 500)
    ref = U.history("stream", 1, 2, slots(500), 128, [300])
    cache = U.to_dev(ref, 500)
    st = torch.cuda.Stream()
    q, k, v = U.new_tokens("stream", 1, 1, 8, 2, 128)
    lens = torch.tensor([300], dtype=torch.int32, device="cuda")
    dq, dk, dv = (U.dev_bf16(x) for x in (q, k, v))
    out = torch.empty_like(dq)
    st.wait_stream(torch.cuda.current_stream())
    attn.kv4_decode(dq, dk, dv, lens, cache, out=out, stream=st)
    kr, vr = torch.empty(2, 1, 2, 301, 128, dtype=torch.bfloat16, device="cuda")
    attn.kv4_read(cache, 0, 301, out=(kr, vr), stream=st)
    st.synchronize()
    tab, pos = K.tables(500, 128, attn.rope_theta), np.array([300])
    ref.write(0, pos, K.rope(k[0], pos, tab), v[0])
    U.close(out[0], *K.attend(K.rope(q[0], pos, tab), pos, ref, 0), "stream")
    assert (K.bf16_to_f64(U.host_bits(kr)) == K.values(ref.codes[0][:, :, :301], ref.scales[0][:, :, :301])).all()


def test_offsets_past_32_bits():
    """A cache of 80 heads of a million slots: the last head's codes lie 5.3 GB in."""
    import torch

    from paper_2607_15865_gb300.kv4 import Kv4Cache
    L, B, Hkv, D = 1 << 20, 10, 8, 128
    attn = context(B, Hkv, Hkv, D, L)
    cache = Kv4Cache.empty(B, Hkv, L, D)
    h = L - 40
    q, k, v = U.new_tokens("far", B, 1, Hkv, Hkv, D)
    dk, dv = U.dev_bf16(k), U.dev_bf16(v)
    lens = torch.tensor([5] * (B - 1) + [h], dtype=torch.int32, device="cuda")
    kc, kvv = U.new_tokens("farc", B, 40, Hkv, Hkv, D)[1:]
    attn.kv4_append(U.dev_bf16(kc), U.dev_bf16(kvv), h, cache)
    out = attn.kv4_decode(U.dev_bf16(q), dk, dv, lens, cache)
    got_k, got_v = attn.kv4_read(cache, h, 40)
    ref = K.Cache(1, Hkv, 64, D)
    tab = K.tables(1, D, attn.rope_theta)
    ang = np.arange(h, L, dtype=np.float64)[:, None] * np.array([attn.rope_theta ** (-2.0 * j / D) for j in range(D // 2)])
    tab = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    b = B - 1
    ref.write(0, np.arange(40), K.rope(kc[b], np.arange(40), tab), kvv[b])
    ref.write(0, np.array([0]), K.rope(k[b], np.array([0]), tab), v[b])
    for t, got in enumerate((got_k, got_v)):
        want = K.values(ref.codes[t][0, :, :40], ref.scales[t][0, :, :40])
        assert (K.bf16_to_f64(U.host_bits(got[b])) == want).all()
    # the history is zeros: h keys of score 0 and value 0, and the new one (slot h)
    kn, vn = K.values(ref.codes[0][0, :, 0], ref.scales[0][0, :, 0]), K.values(ref.codes[1][0, :, 0], ref.scales[1][0, :, 0])
    s = (K.bf16_to_f64(K.rope(q[b], np.array([0]), tab))[0] * kn).sum(-1) / np.sqrt(D)
    w = np.exp(s) / (np.exp(s) + h)
    U.close(out[b, 0], w[:, None] * vn, np.abs(w[:, None] * vn), "far")


# ------------------------------------------------------------------ refusals

def test_refusals():
    import torch

    from paper_2607_15865_gb300 import _lib
    from paper_2607_15865_gb300.kv4 import Kv4Cache
    attn = context(1, 4, 2, 64, 100)
    cache = attn.kv4_cache()
    q, k, v = (U.dev_bf16(x) for x in U.new_tokens("ref", 1, 4, 4, 2, 64))
    lens = torch.tensor([3], dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    for bad in (dict(hist_len=97), dict(hist_len=-1)):
        with pytest.raises(_lib.AttnError):
            attn.kv4_append(k, v, cache=cache, **bad)
        with pytest.raises((_lib.AttnError, TypeError)):
            attn.kv4_prefill_kv(q, k, v, cache=cache, **bad)
    for first, count in ((-1, 2), (0, 101), (100, 1), (0, -1)):
        with pytest.raises(_lib.AttnError):
            attn.kv4_read(cache, first, count)
    with pytest.raises(ValueError):
        attn.kv4_append(k[:, :, :1], v, 0, cache)                      # shape
    with pytest.raises(ValueError):
        attn.kv4_append(k.transpose(1, 2).contiguous().transpose(1, 2), v, 0, cache)  # strides
    with pytest.raises(TypeError):
        attn.kv4_append(k.float(), v, 0, cache)
    with pytest.raises(TypeError):
        attn.kv4_decode(q, k, v, lens.long(), cache)
    with pytest.raises(TypeError):
        attn.kv4_decode(q, k, v, lens, cache.k_codes)
    with pytest.raises(ValueError):
        attn.kv4_decode(q, k, v, lens, Kv4Cache.empty(1, 2, 99, 64))   # another max_len
    with pytest.raises(ValueError):
        attn.kv4_decode(q, k, v, lens, Kv4Cache.empty(1, 2, 100, 128))
    with pytest.raises(TypeError):
        attn.kv4_prefill_kv(q, k, v, 0, cache, torch.empty(attn.kv4_workspace(4) - 1, dtype=torch.uint8, device="cuda"))
    q17, k17, v17 = (U.dev_bf16(x) for x in U.new_tokens("ref", 1, 17, 4, 2, 64))
    with pytest.raises(_lib.AttnError):
        attn.kv4_decode(q17, k17, v17, lens, cache)
    c = [t.clone() for t in before]
    with pytest.raises(ValueError):
        Kv4Cache(200, *c)
    with pytest.raises(TypeError):
        Kv4Cache(100, c[0], c[1].float(), c[2], c[3])
    with pytest.raises(ValueError):
        Kv4Cache(100, c[0].transpose(2, 3), c[1], c[2], c[3])
    odd = torch.empty(c[0].numel() + 1, dtype=torch.uint8, device="cuda")[1:].view(c[0].shape)
    with pytest.raises(_lib.AttnError):
        attn.kv4_append(k, v, 0, Kv4Cache(100, odd, c[1], c[2], c[3]))  # 16-byte alignment
    torch.cuda.synchronize()
    assert all((x == y).all() for x, y in zip(before, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)))
    assert attn.device_error() == 0
