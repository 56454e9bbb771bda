"""The 4-bit KV cache, as cases to be timed and compared: quantising new keys and values as they are
written, reading slots back, and the decode and prefill_kv stages over such a cache.

A cache of max_len slots holds, per sequence and kv head, `codes` uint8 [B, Hkv, Lp, D / 2] and `scales`
int16 [B, Hkv, Lp, D / 32] for k and the same for v (Lp: max_len rounded up to a multiple of 64).  The D
values of a slot are in groups of 32; a group x has
  range     lo = min(x, 0), hi = max(x, 0)
  scale     s, the smallest number of 4 significant bits that is >= (hi - lo) / 15, at least 2^-126
  zero      z = rint(-lo / s)                              (rint: to nearest, ties to even)
  code      c = min(max(rint(x / s) + z, 0), 15)
  value     (c - z) s, which is a bf16 exactly
and a group with an infinity or a NaN has c = z = 0 and a NaN for s.  `scales` holds s as a bf16 whose
four lowest bits, zero in s, are z.  A 32-bit word of `codes` holds 8 values, the code of value j at bit
(0, 16, 4, 20, 8, 24, 12, 28)[j].

Keys are quantised after RoPE, from the bf16 that the bf16 cache would hold.  What attends to a token sees
the values that the cache holds for it, its own included.

Kinds (the "kind" of a case):
  append   a chunk of `chunk` new tokens written at slot `hist`, and read back
  read     slots `first` .. `first + count - 1` read back
  decode   `n` new tokens per sequence over histories of up to `hist` tokens
  prefill  a chunk of `chunk` new tokens over `hist` cached ones
"""
import functools
import math

import torch

own = False
DEV = "cuda"
NIBBLES = (0, 16, 4, 20, 8, 24, 12, 28)
GROUP = 32

# (query heads, kv heads, head_dim, rope theta): the shapes of the framework's workloads and tests
TINY = dict(hq=4, hkv=2, d=64, theta=1.0e4)
SMALL64 = dict(hq=32, hkv=8, d=64, theta=5.0e5)
GQA7 = dict(hq=28, hkv=4, d=128, theta=1.0e6)
GQA4 = dict(hq=32, hkv=8, d=128, theta=5.0e5)
GQA5 = dict(hq=40, hkv=8, d=128, theta=1.0e6)
GQA16 = dict(hq=32, hkv=2, d=128, theta=1.0e6)
MHA = dict(hq=8, hkv=8, d=128, theta=1.0e4)


def listed():
    return [
        # the tiny chain's chunk of a prompt: the smallest write
        dict(name="append_8_d64", kind="append", b=1, L=32, hist=16, chunk=8, **TINY),
        # the last segment of a 32K prompt
        dict(name="append_4096_over_28672", kind="append", b=1, L=32768, hist=28672, chunk=4096, **GQA5),
        # a conversation's history for a user that attends in bf16
        dict(name="read_2048", kind="read", b=1, L=2048, first=0, count=2048, **GQA4),
        # one layer of a long session, a ragged number of slots
        dict(name="read_32767", kind="read", b=1, L=32768, first=0, count=32767, **GQA5),
        # a step of one short conversation: latency
        dict(name="decode_b1_1024", kind="decode", b=1, L=8192, hist=1024, n=1, mixed=False, **GQA4),
        # a step of one long conversation
        dict(name="decode_b1_32767", kind="decode", b=1, L=32768, hist=32767, n=1, mixed=False, **GQA5),
        # a step of a serving batch, sequences of mixed lengths
        dict(name="decode_b16_mixed", kind="decode", b=16, L=8192, hist=8183, n=1, mixed=True, **GQA4),
        # four draft tokens verified over an 8K history
        dict(name="verify_4_over_8188", kind="decode", b=1, L=8192, hist=8188, n=4, mixed=False, **GQA4),
        # five draft tokens of three sequences of a small model
        dict(name="verify_5_d64_b3", kind="decode", b=3, L=4096, hist=4001, n=5, mixed=True, **SMALL64),
        # the next message of a conversation
        dict(name="prefill_512_over_1536", kind="prefill", b=1, L=2048, hist=1536, chunk=512, **GQA4),
        # a short ragged message over a longer history, two sequences
        dict(name="prefill_77_over_5000_b2", kind="prefill", b=2, L=8192, hist=5000, chunk=77, **GQA7),
        # the last segment of a 32K prompt, its attention
        dict(name="prefill_4096_over_28672", kind="prefill", b=1, L=32768, hist=28672, chunk=4096, **GQA5),
    ]


def _log(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["append", "read", "decode", "decode", "decode", "prefill"])
    shape = dict(rng.choice([TINY, SMALL64, GQA7, GQA4, GQA5, GQA16, MHA]))
    b = rng.choice([1, 1, 2, 3, 4, 8, 16])
    most = 32767 if b <= 2 else 8191
    if kind == "append":
        chunk = _log(rng, 1, 4096 // b)
        hist = rng.choice([0, _log(rng, 1, most)])
        return dict(kind=kind, b=b, L=hist + chunk + rng.randint(0, 64), hist=hist, chunk=chunk, **shape)
    if kind == "read":
        count = _log(rng, 1, min(most, 65536 // b))
        first = rng.choice([0, rng.randint(0, 300)])
        return dict(kind=kind, b=b, L=first + count + rng.randint(0, 64), first=first, count=count, **shape)
    if kind == "decode":
        hist = _log(rng, 1, most)
        n = rng.choice([1, 1, 1, rng.randint(2, 8), 16])
        return dict(kind=kind, b=b, L=hist + n + rng.randint(0, 64), hist=hist, n=n, mixed=b > 1 and rng.random() < 0.7,
                    **shape)
    b = min(b, 4)
    chunk = _log(rng, 1, 4096 // b)
    hist = rng.choice([0, _log(rng, 1, 16384 // b)])
    return dict(kind=kind, b=b, L=hist + chunk + rng.randint(0, 64), hist=hist, chunk=chunk, **shape)


def _lengths(c):
    """The batch's history lengths: all `hist`, or spread over 0 .. hist."""
    if not c["mixed"]:
        return [c["hist"]] * c["b"]
    return [c["hist"]] + [int(c["hist"] * ((i * 0.61803) % 1.0)) for i in range(1, c["b"])]


# ------------------------------------------------------------------ the plain form

def _rope(x, cos, sin):
    """x [..., D] float at the positions of cos and sin [..., D / 2]: element j turns with j + D / 2."""
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16).float()


def _quantise(x):
    """x [..., D] float -> codes [..., D / 2] uint8, scales [..., D / 32] int16."""
    g = x.unflatten(-1, (-1, GROUP))
    finite = torch.isfinite(g).all(-1)
    lo, hi = g.amin(-1).clamp(max=0.0), g.amax(-1).clamp(min=0.0)
    # the divisor as a tensor: torch multiplies by the reciprocal of a number, which is not the same
    bits = ((hi * 0.5 - lo * 0.5) / torch.full_like(lo, 7.5)).view(torch.int32)
    bits = (bits + 0xFFFFF) & -0x100000
    # one step up where a difference that float rounds off leaves hi - lo above 15 s
    bits += (hi * 0.5 - bits.view(torch.float32) * 7.5 > lo * 0.5).int() << 20
    s = bits.view(torch.float32).clamp(min=2.0 ** -126)
    z = torch.round(-lo / s)
    c = (torch.round(g / s[..., None]) + z[..., None]).clamp(0, 15)
    c = torch.where(finite[..., None], c, torch.zeros_like(c)).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 8))
    z = torch.where(finite, z, torch.zeros_like(z))
    s = torch.where(finite, s.view(torch.int32) >> 16, torch.full_like(bits, 0x7FF0))
    return (c[..., [0, 4, 1, 5]] | (c[..., [2, 6, 3, 7]] << 4)).flatten(-2), (s | z.int()).to(torch.int16)


def _values(codes, scales):
    """The float values [..., D] that codes and scales stand for."""
    w = codes.unflatten(-1, (-1, 4))
    c = torch.cat([w & 15, w >> 4], -1)[..., [0, 2, 4, 6, 1, 3, 5, 7]].flatten(-2).unflatten(-1, (-1, GROUP)).float()
    m = scales.int()
    s = ((m & 0x7FF0) << 16).view(torch.float32)
    return ((c - (m & 15).float()[..., None]) * s[..., None]).flatten(-2)


def _write(st, pos):
    """New keys and values quantised into slots pos [B, n] of the state's cache."""
    k = _rope(st["k"].float(), st["cos"][pos][:, :, None], st["sin"][pos][:, :, None])
    rows = torch.arange(pos.shape[0], device=DEV)[:, None]
    for x, name in ((k, "k"), (st["v"].float(), "v")):
        codes, scales = _quantise(x)
        st[name + "_codes"][rows, :, pos] = codes
        st[name + "_scales"][rows, :, pos] = scales


def _attend(st, pos, slots):
    """Causal attention of q [B, n, Hq, D] at positions pos [B, n] over slots 0 .. slots - 1."""
    b, n, hq, d = st["q"].shape
    k = _values(st["k_codes"][:, :, :slots], st["k_scales"][:, :, :slots])
    v = _values(st["v_codes"][:, :, :slots], st["v_scales"][:, :, :slots])
    hkv = k.shape[1]
    q = _rope(st["q"].float(), st["cos"][pos][:, :, None], st["sin"][pos][:, :, None])
    q = q.transpose(1, 2).reshape(b, hkv, -1, d)
    p = q @ k.transpose(2, 3)
    p *= d ** -0.5
    hidden = torch.arange(slots, device=DEV) > pos[:, :, None]  # [B, n, slots]
    p = p.view(b, hq, n, slots).masked_fill_(hidden[:, None], -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    p = p.view(b, hkv, -1, slots)
    out = (p @ v) / p.sum(-1, keepdim=True)
    return out.view(b, hq, n, d).transpose(1, 2).contiguous().to(torch.bfloat16)


# ------------------------------------------------------------------ states

class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed)

    def __call__(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV)


def _given(c, seed):
    """The inputs of a case: bf16 activations of unit size, keys with a few channels far from zero (as the
    keys of trained models have them), a cache whose every slot holds some token."""
    r = _Rand(seed)
    b, hq, hkv, d, slots = c["b"], c["hq"], c["hkv"], c["d"], (c["L"] + 63) // 64 * 64
    shift = 2.0 * r(hkv, d) * (r(hkv, d) > 1.3)
    st = {}
    if c["kind"] != "append":
        for name in ("k", "v"):
            x = r(b, hkv, slots, d)
            if name == "k":
                x += shift[:, None]
            st[name + "_codes"], st[name + "_scales"] = _quantise(x.to(torch.bfloat16).float())
    else:
        st = {x + y: torch.zeros((b, hkv, slots, w), dtype=t, device=DEV) for x in "kv"
              for y, w, t in (("_codes", d // 2, torch.uint8), ("_scales", d // GROUP, torch.int16))}
    n = c.get("n", c.get("chunk", 0))
    if n:
        st["q"] = (1.3 * r(b, n, hq, d)).to(torch.bfloat16)
        st["k"] = (r(b, n, hkv, d) + shift).to(torch.bfloat16)
        st["v"] = r(b, n, hkv, d).to(torch.bfloat16)
    if c["kind"] == "decode":
        st["hist"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    return st


def _tables(c, dtype):
    ang = torch.arange(c["L"], dtype=torch.float64, device=DEV)[:, None] * torch.tensor(
        [c["theta"] ** (-2.0 * j / c["d"]) for j in range(c["d"] // 2)], dtype=torch.float64, device=DEV)
    return ang.cos().to(dtype), ang.sin().to(dtype)


@functools.lru_cache(maxsize=32)
def _handle(b, hq, hkv, d, L, theta):
    """The context of an attention shape, which a program makes once."""
    from paper_2607_15865_gb300.attention import Attention
    return Attention(b, hq, hkv, d, L, theta)


def prepare(case, seed):
    st = dict(_given(case, seed), case=case)
    if own:
        from paper_2607_15865_gb300.kv4 import Kv4Cache
        st["attn"] = _handle(*(case[x] for x in ("b", "hq", "hkv", "d", "L", "theta")))
        st["cache"] = Kv4Cache(case["L"], *(st[x] for x in ("k_codes", "k_scales", "v_codes", "v_scales")))
        if case["kind"] == "prefill":
            size = st["attn"].kv4_workspace(case["hist"] + case["chunk"])
            st["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    else:
        st["cos"], st["sin"] = _tables(case, torch.float32)
    return st


# What the stages write besides their output: the packed cache itself, compared bit for bit (the arithmetic of
# the quantiser is exact, so two right ones agree in every code).
def _with_cache(out, st):
    return {"out": out, **{x: st[x] for x in ("k_codes", "k_scales", "v_codes", "v_scales")}}


def run(st):
    c = st["case"]
    kind = c["kind"]
    if own:
        attn, cache = st["attn"], st["cache"]
        if kind == "append":
            attn.kv4_append(st["k"], st["v"], c["hist"], cache)
            return attn.kv4_read(cache, c["hist"], c["chunk"])
        if kind == "read":
            return attn.kv4_read(cache, c["first"], c["count"])
        if kind == "decode":
            return _with_cache(attn.kv4_decode(st["q"], st["k"], st["v"], st["hist"], cache), st)
        return _with_cache(attn.kv4_prefill_kv(st["q"], st["k"], st["v"], c["hist"], cache, st["workspace"]), st)
    if kind == "decode":
        pos = st["hist"].long()[:, None] + torch.arange(c["n"], device=DEV)
        _write(st, pos)
        return _with_cache(_attend(st, pos, c["hist"] + c["n"]), st)
    if kind != "read":
        pos = torch.arange(c["hist"], c["hist"] + c["chunk"], device=DEV).expand(c["b"], -1)
        _write(st, pos)
    if kind == "prefill":
        return _with_cache(_attend(st, pos, c["hist"] + c["chunk"]), st)
    lo, n = (c["first"], c["count"]) if kind == "read" else (c["hist"], c["chunk"])
    return tuple(_values(st[x + "_codes"][:, :, lo:lo + n], st[x + "_scales"][:, :, lo:lo + n]).to(torch.bfloat16)
                 for x in "kv")


def work(case):
    c = case
    b, hq, hkv, d, kind = c["b"], c["hq"], c["hkv"], c["d"], c["kind"]
    packed, plain = 2 * hkv * (d // 2 + d // 16), 2 * hkv * d * 2  # bytes of a token's k and v in both forms
    if kind == "append":
        n = b * c["chunk"]
        return {"bytes": n * (2 * plain + packed) + c["chunk"] * d * 4, "flops": 0}
    if kind == "read":
        return {"bytes": b * c["count"] * (plain + packed), "flops": 0}
    n = c["n"] if kind == "decode" else c["chunk"]
    lens = _lengths(c) if kind == "decode" else [c["hist"]] * b
    pairs = sum(n * h + n * (n + 1) // 2 for h in lens)
    rows = n * b * (2 * hq * d * 2 + plain)  # q, out, k and v of the new tokens
    return {"bytes": rows + packed * sum(h + n for h in lens), "flops": 4.0 * d * hq * pairs}


# ------------------------------------------------------------------ in 64 bits

def _exact_quantised(x):
    """The values (float64) that stand for x [..., D], straight from the definition at the top."""
    g = x.double().reshape(x.shape[:-1] + (-1, GROUP))
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    lo, hi = torch.minimum(g.min(-1, True).values, zero), torch.maximum(g.max(-1, True).values, zero)
    m, e = torch.frexp((hi - lo) / 15.0)
    s = torch.maximum(torch.ldexp(torch.ceil(m * 16.0) / 16.0, e), zero + 2.0 ** -126)
    z = torch.round(-lo / s)
    c = torch.minimum(torch.maximum(torch.round(g / s) + z, zero), zero + 15.0)
    return ((c - z) * s).reshape(x.shape)


def _exact_stored(codes, scales):
    words = codes.contiguous().view(torch.int32)
    c = torch.stack([(words >> sh) & 15 for sh in NIBBLES], -1).double().flatten(-2)
    m = scales.contiguous()
    s = (m & 0x7FF0).view(torch.bfloat16).double()
    z = (m & 15).double()
    return (c - z.repeat_interleave(GROUP, -1)) * s.repeat_interleave(GROUP, -1)


def _exact_turned(x, pos, c):
    """RoPE in 64 bits of x [n, H, D] at positions pos [n], rounded to the bf16 that the stages use."""
    cos, sin = (t[pos][:, None] for t in _tables(c, torch.float64))
    turned = torch.view_as_complex(torch.stack(x.double().chunk(2, -1), -1).contiguous()) * torch.complex(cos, sin)
    return torch.cat([turned.real, turned.imag], -1).to(torch.bfloat16).double()


def exact(case, seed):
    c, st = case, _given(case, seed)
    kind = c["kind"]
    if kind == "read":
        at = slice(c["first"], c["first"] + c["count"])
        return tuple(_exact_stored(st[x + "_codes"][:, :, at], st[x + "_scales"][:, :, at]) for x in "kv")
    n = c["n"] if kind == "decode" else c["chunk"]
    lens = _lengths(c) if kind == "decode" else [c["hist"]] * c["b"]
    new_k, new_v, outs = [], [], []
    for b, hist in enumerate(lens):
        pos = torch.arange(hist, hist + n, device=DEV)
        new_k.append(_exact_quantised(_exact_turned(st["k"][b], pos, c)).transpose(0, 1))
        new_v.append(_exact_quantised(st["v"][b]).transpose(0, 1))
        if kind == "append":
            continue
        q, heads = _exact_turned(st["q"][b], pos, c), []
        for h in range(c["hq"]):
            g = h // (c["hq"] // c["hkv"])
            k, v = (torch.cat([_exact_stored(st[x + "_codes"][b, g, :hist], st[x + "_scales"][b, g, :hist]), y[b][g]])
                    for x, y in (("k", new_k), ("v", new_v)))
            a = (q[:, h] @ k.T) / math.sqrt(c["d"])
            a = torch.where(torch.arange(hist + n, device=DEV) <= pos[:, None], a, -math.inf)
            heads.append(torch.softmax(a, -1) @ v)
        outs.append(torch.stack(heads, 1))
    if kind == "append":
        return torch.stack(new_k), torch.stack(new_v)
    return {"out": torch.stack(outs), "k_codes": None, "k_scales": None, "v_codes": None, "v_scales": None}
