"""Attention with a sliding window and first tokens that stay visible, and the verification of a tree of drafted
tokens over the KV cache, as cases to be timed and compared.

Caches are bf16 [B, Hkv, L, D]; a token's k is held after RoPE (element j turns with j + D / 2, the angle of position p
is p theta^(-2j/D)), rounded to bf16, as is the rotated q.  Query head h reads kv head h / (Hq / Hkv).  A query at
position p sees the slots s <= p with p - s < window or s < sinks (window 0: all of them).

Kinds (the "kind" of a case):
  window_prefill  a chunk of `chunk` new tokens of every sequence over `hist` cached ones
  window_decode   `n` new tokens per sequence, one after the other, over histories of up to `hist` tokens
  tree_decode     a tree of up to `n` drafted tokens per sequence over histories of up to `hist` tokens.  Token i has
                  the parent parents[b, i] < i (-1: it follows the history; -2: there is no token i), lies in slot
                  hist + i, is at position hist + its depth, and sees the history, its ancestors and itself, as far as
                  the window of their positions allows
  tree_accept     token leaf[b] of such a tree and its ancestors (-1: none) are accepted: their k and v move, in order,
                  to the slots from hist on, in the caches of `layers` layers; the new lengths
"""
import functools
import math

import torch

own = False
DEV = "cuda"

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
        # the tiny chain's follow-up, a window shorter than its history: the smallest call
        dict(name="window_prefill_8_over_16_d64", kind="window_prefill", b=1, L=32, hist=16, chunk=8, window=12, sinks=2,
             **TINY),
        # a short ragged message over a longer history, two sequences
        dict(name="window_prefill_77_over_5000_b2", kind="window_prefill", b=2, L=8192, hist=5000, chunk=77, window=1000,
             sinks=4, **GQA7),
        # the last segment of a 32K prompt
        dict(name="window_prefill_4096_over_28672", kind="window_prefill", b=1, L=32768, hist=28672, chunk=4096,
             window=4096, sinks=4, **GQA5),
        # a step of one conversation over an 8K history: latency
        dict(name="window_decode_b1_8191", kind="window_decode", b=1, L=8192, hist=8191, n=1, window=1024, sinks=4,
             mixed=False, **GQA4),
        # a step of a serving batch, sequences of mixed lengths
        dict(name="window_decode_b16_mixed", kind="window_decode", b=16, L=8192, hist=8183, n=1, window=4096, sinks=4,
             mixed=True, **GQA4),
        # five draft tokens of three sequences of a small model
        dict(name="window_decode_5_d64_b3", kind="window_decode", b=3, L=4096, hist=4001, n=5, window=512, sinks=16,
             mixed=True, **SMALL64),
        # a small tree after a short conversation: latency
        dict(name="tree_decode_8_over_1024", kind="tree_decode", b=1, L=8192, hist=1024, n=8, width=3, window=0, sinks=0,
             mixed=False, **GQA4),
        # the largest tree at the end of a long session
        dict(name="tree_decode_64_over_32700", kind="tree_decode", b=1, L=32768, hist=32700, n=64, width=16, window=0,
             sinks=0, mixed=False, **GQA5),
        # trees of a serving batch, mixed lengths and numbers of tokens
        dict(name="tree_decode_12_b16_mixed", kind="tree_decode", b=16, L=8192, hist=8180, n=12, width=4, window=0,
             sinks=0, mixed=True, **GQA4),
        # trees of a small model whose layer has a window
        dict(name="tree_decode_26_d64_b3_window", kind="tree_decode", b=3, L=4096, hist=4001, n=26, width=6, window=1024,
             sinks=4, mixed=True, **SMALL64),
        # one layer of one short tree
        dict(name="tree_accept_8", kind="tree_accept", b=1, L=1040, hist=1024, n=8, width=3, layers=1, mixed=False, **GQA4),
        # every layer of a small batch
        dict(name="tree_accept_64_b4_32_layers", kind="tree_accept", b=4, L=640, hist=560, n=64, width=16, layers=32,
             mixed=True, **GQA4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["window_prefill", "window_prefill", "window_decode", "window_decode", "tree_decode", "tree_decode",
                       "tree_decode", "tree_accept"])
    shape = dict(rng.choice([TINY, SMALL64, GQA7, GQA4, GQA5, GQA16, MHA]))
    sinks = rng.choice([0, 1, 4, _log(rng, 2, 300)])
    if kind == "window_prefill":
        b = rng.choice([1, 1, 2, 3, 4])
        chunk = _log(rng, 1, 4096 // b)
        hist = rng.choice([0, _log(rng, 1, 28672 // b)])
        return dict(kind=kind, b=b, L=hist + chunk + rng.randint(0, 64), hist=hist, chunk=chunk, window=_log(rng, 1, 4096),
                    sinks=sinks, **shape)
    b = rng.choice([1, 1, 2, 3, 4, 8, 16])
    mixed = b > 1 and rng.random() < 0.7
    if kind == "tree_accept":
        n, hist = _log(rng, 1, 64), _log(rng, 1, 560)
        return dict(kind=kind, b=b, L=hist + n + rng.randint(0, 16), hist=hist, n=n, width=rng.randint(1, 16),
                    layers=_log(rng, 1, max(1, 128 // b) if b > 4 else 32), mixed=mixed, **shape)
    hist = _log(rng, 1, 32700 if b <= 2 else 8191)
    if kind == "window_decode":
        n = rng.choice([1, 1, rng.randint(2, 16), _log(rng, 1, 64)])
        return dict(kind=kind, b=b, L=hist + n + rng.randint(0, 64), hist=hist, n=n, window=_log(rng, 1, 8192), sinks=sinks,
                    mixed=mixed, **shape)
    n = _log(rng, 1, 64)
    window = rng.choice([0, 0, _log(rng, 1, 8192)])
    return dict(kind=kind, b=b, L=hist + n + rng.randint(0, 64), hist=hist, n=n, width=rng.randint(1, 16), window=window,
                sinks=sinks if window else 0, mixed=mixed, **shape)


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
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)


def _visible(pos, key_pos, c):
    """Whether a query at `pos` sees a key at `key_pos` that is not after it (tensors that broadcast)."""
    if c["window"] == 0:
        return key_pos <= pos
    return (key_pos <= pos) & ((pos - key_pos < c["window"]) | (key_pos < c["sinks"]))


def _attend(q, k, v, seen):
    """q [B, n, Hq, D] bf16, k and v [B, Hkv, slots, D] bf16, seen [B or 1, n, slots] -> [B, n, Hq, D] bf16."""
    b, n, hq, d = q.shape
    hkv, slots = k.shape[1], k.shape[2]
    q = q.float().transpose(1, 2).reshape(b, hkv, -1, d)
    p = q @ k.float().transpose(2, 3)
    p *= d ** -0.5
    p = p.view(b, hq, n, slots).masked_fill_(~seen[:, None], -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    p = p.view(b, hkv, -1, slots)
    out = (p @ v.float()) / p.sum(-1, keepdim=True)
    return out.view(b, hq, n, d).transpose(1, 2).contiguous().to(torch.bfloat16)


def _window_prefill(st, c):
    hist, n, end = c["hist"], c["chunk"], c["hist"] + c["chunk"]
    cos, sin = (st[x][hist:end][:, None] for x in ("cos", "sin"))
    st["k_cache"][:, :, hist:end] = _rope(st["k"].float(), cos, sin).transpose(1, 2)
    st["v_cache"][:, :, hist:end] = st["v"].transpose(1, 2)
    q = _rope(st["q"].float(), cos, sin)
    lo = max(0, hist - c["window"] + 1)
    head = min(c["sinks"], lo)
    slots = torch.cat([torch.arange(head, device=DEV), torch.arange(lo, end, device=DEV)])
    k, v = (torch.cat([st[x][:, :, :head], st[x][:, :, lo:end]], 2) for x in ("k_cache", "v_cache"))
    pos = torch.arange(hist, end, device=DEV)
    return _attend(q, k, v, _visible(pos[:, None], slots, c)[None])


def _ancestry(parents):
    """parents [B, n] -> whether token j is i or an ancestor of i [B, n, n], as far as there is a token i."""
    b, n = parents.shape
    up = torch.nn.functional.one_hot(parents.long().clamp(min=-1) + 1, n + 1)[..., 1:].float()
    reach = up + torch.eye(n, device=DEV)
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (reach @ reach).clamp(max=1.0)
    return (reach > 0) & (parents >= -1)[..., None]


def _new_tokens(st, c, family, depth, there):
    """Drafted tokens written to their slots, and their attention over those and the history."""
    n, lens = c["n"], st["hist"].long()
    b = lens.shape[0]
    pos = (lens[:, None] + depth).clamp(max=c["L"] - 1)
    cos, sin = (st[x][pos][:, :, None] for x in ("cos", "sin"))
    k, q = _rope(st["k"].float(), cos, sin), _rope(st["q"].float(), cos, sin)
    rows, at = torch.arange(b, device=DEV)[:, None].expand(b, n), lens[:, None] + torch.arange(n, device=DEV)
    for x, new in (("k_cache", k), ("v_cache", st["v"])):
        st[x][rows[there], :, at[there]] = new[there]
    slots = c["hist"] + n
    s = torch.arange(slots, device=DEV)
    seen = (s < lens[:, None])[:, None] & _visible(pos[:, :, None], s, c)
    mine = family & _visible(pos[:, :, None], pos[:, None], c)
    bb, ii, jj = mine.nonzero(as_tuple=True)
    seen[bb, ii, lens[bb] + jj] = True
    seen[..., 0] |= ~there  # (a row of no token, which is not an output, needs some key)
    out = _attend(q, st["k_cache"][:, :, :slots], st["v_cache"][:, :, :slots], seen)
    st["out"][there] = out[there]
    return st["out"]


def _accept(st, c):
    b, n, lens = c["b"], c["n"], st["hist"].long()
    family = _ancestry(st["parents"])
    leaf = st["leaf"].long()
    path = family[torch.arange(b, device=DEV), leaf.clamp(min=0)] & (leaf >= 0)[:, None]
    bb, src = path.nonzero(as_tuple=True)
    dst = (path.cumsum(-1) - 1)[bb, src]
    for k, v in st["caches"]:
        for x in (k, v):
            x[bb, :, lens[bb] + dst] = x[bb, :, lens[bb] + src]
    st["new_len"].copy_(lens + path.sum(-1))


# ------------------------------------------------------------------ states

def _rand(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _given(c, seed):
    """The inputs of a case: bf16 activations of unit size, keys with a few channels far from zero (as the keys of
    trained models have them), a cache whose every slot holds some token, trees that are `width` tokens wide or so."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    b, hq, hkv, d, kind = c["b"], c["hq"], c["hkv"], c["d"], c["kind"]
    shift = 2.0 * _rand(g, hkv, d) * (_rand(g, hkv, d) > 1.3)
    layers = c.get("layers", 1)
    pool = torch.empty((layers, 2, b, hkv, c["L"], d), dtype=torch.bfloat16, device=DEV)
    for kv in pool:
        kv[0] = _rand(g, b, hkv, c["L"], d) + shift[:, None]
        kv[1] = _rand(g, b, hkv, c["L"], d)
    st = {"pool": pool, "caches": [(kv[0], kv[1]) for kv in pool], "k_cache": pool[0, 0], "v_cache": pool[0, 1]}
    n = c.get("n", c.get("chunk", 0))
    if kind != "tree_accept":
        st["q"] = (1.3 * _rand(g, b, n, hq, d)).to(torch.bfloat16)
        st["k"] = (_rand(g, b, n, hkv, d) + shift).to(torch.bfloat16)
        st["v"] = _rand(g, b, n, hkv, d).to(torch.bfloat16)
        st["out"] = torch.zeros_like(st["q"])
    if kind != "window_prefill":
        st["hist"] = torch.tensor(_lengths(c), dtype=torch.int32, device=DEV)
    if kind.startswith("tree"):
        i = torch.arange(n, device=DEV).expand(b, n)
        back = (torch.rand((b, n), generator=g, device=DEV) * c["width"]).long()
        parents = torch.maximum(i - 1 - back, torch.where(i == 0, -1, 0))
        if c["mixed"]:  # trees of other numbers of tokens
            count = n - (torch.rand((b, 1), generator=g, device=DEV) * (n / 2)).long()
            parents = torch.where(i < count, parents, -2)
        else:
            count = torch.full((b, 1), n, device=DEV)
        st["parents"] = parents.to(torch.int32).contiguous()
        if kind == "tree_accept":
            st["leaf"] = ((torch.rand((b, 1), generator=g, device=DEV) * (count + 1)).long() - 1)[:, 0].to(torch.int32)
            st["new_len"] = torch.zeros_like(st["leaf"])
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
        st["attn"] = _handle(*(case[x] for x in ("b", "hq", "hkv", "d", "L", "theta")))
    elif case["kind"] != "tree_accept":
        st["cos"], st["sin"] = _tables(case, torch.float32)
    return st


def run(st):
    c = st["case"]
    kind = c["kind"]
    caches = [st["k_cache"], st["v_cache"]]
    if kind == "tree_accept":
        if own:
            st["attn"].tree_accept(st["hist"], st["parents"], st["leaf"], st["caches"], new_len=st["new_len"])
        else:
            _accept(st, c)
        return {"new_len": st["new_len"], "caches": st["pool"]}
    if own:
        attn, new = st["attn"], (st["q"], st["k"], st["v"])
        if kind == "window_prefill":
            out = attn.window_prefill_kv(*new, c["hist"], c["window"], *caches, sinks=c["sinks"], out=st["out"])
        elif kind == "window_decode":
            out = attn.window_decode(*new, st["hist"], c["window"], *caches, sinks=c["sinks"], out=st["out"])
        else:
            out = attn.tree_decode(*new, st["hist"], st["parents"], *caches, window=c["window"], sinks=c["sinks"],
                                   out=st["out"])
    elif kind == "window_prefill":
        out = _window_prefill(st, c)
    elif kind == "window_decode":
        i = torch.arange(c["n"], device=DEV)
        out = _new_tokens(st, c, (i <= i[:, None]).expand(c["b"], -1, -1), i.expand(c["b"], -1),
                          torch.ones((c["b"], c["n"]), dtype=torch.bool, device=DEV))
    else:
        family = _ancestry(st["parents"])
        out = _new_tokens(st, c, family, (family.sum(-1) - 1).clamp(min=0), st["parents"] >= -1)
    return {"out": out, "k_cache": caches[0], "v_cache": caches[1]}


def _pairs(lo, hi, window, sinks):
    """Slots that the queries at positions lo .. hi - 1 see, all together, and by any of them."""
    if window == 0:
        window = hi
    total = 0
    for p in range(lo, hi):
        start = max(0, p - window + 1)
        total += p - start + 1 + min(sinks, start)
    first = max(0, lo - window + 1)
    return total, hi - first + min(sinks, first)


def work(case):
    c = case
    b, hq, hkv, d, kind = c["b"], c["hq"], c["hkv"], c["d"], c["kind"]
    row = 2 * hkv * d * 2  # bytes of a token's k and v
    if kind == "tree_accept":  # of a path of about the mean length, read and written
        return {"bytes": c["layers"] * b * (1 + c["n"] // (c["width"] + 2)) * 2 * row, "flops": 0}
    n = c.get("n", c.get("chunk", 0))
    total = slots = 0
    for h in ([c["hist"]] * b if kind == "window_prefill" else _lengths(c)):
        t, s = _pairs(h, h + n, c["window"], c["sinks"])
        if kind == "tree_decode":  # a drafted token sees a few of the others: its ancestors
            t -= n * (n + 1) // 2 - n * min(n, 1 + n // (c["width"] + 1))
        total, slots = total + t, slots + s
    return {"bytes": b * n * (2 * hq * d * 2 + row) + slots * row, "flops": 4.0 * d * hq * total}


# ------------------------------------------------------------------ in 64 bits

def _exact_turned(x, pos, c):
    """RoPE in 64 bits of x [n, H, D] at positions pos [n], rounded to the bf16 that the stages use."""
    cos, sin = (t[pos][:, None] for t in _tables(c, torch.float64))
    turned = torch.view_as_complex(torch.stack(x.double().chunk(2, -1), -1).contiguous()) * torch.complex(cos, sin)
    return torch.cat([turned.real, turned.imag], -1).to(torch.bfloat16).double()


def _exact_trees(c, st):
    """Per sequence, for each token its ancestors and itself in order (none where there is no token)."""
    trees = []
    for row in st["parents"].tolist():
        chains = []
        for i, p in enumerate(row):
            chains.append([] if p == -2 else (chains[p] if p >= 0 else []) + [i])
        trees.append(chains)
    return trees


def exact(case, seed):
    c, st = case, _given(case, seed)
    kind, window, sinks = c["kind"], c.get("window", 0), c.get("sinks", 0)
    if kind == "tree_accept":
        old, caches, lens = st["pool"], st["pool"].double(), []
        for b, (h, leaf, chains) in enumerate(zip(_lengths(c), st["leaf"].tolist(), _exact_trees(c, st))):
            path = chains[leaf] if leaf >= 0 else []
            lens.append(h + len(path))
            for j, i in enumerate(path):
                caches[:, :, b, :, h + j] = old[:, :, b, :, h + i].double()
        return {"new_len": torch.tensor(lens, dtype=torch.int32, device=DEV), "caches": caches}
    n = c.get("n", c.get("chunk", 0))
    lens = [c["hist"]] * c["b"] if kind == "window_prefill" else _lengths(c)
    trees = _exact_trees(c, st) if kind == "tree_decode" else None
    out = torch.zeros((c["b"], n, c["hq"], c["d"]), dtype=torch.float64, device=DEV)
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    for b, h in enumerate(lens):
        first = max(0, h - window + 1) if window else 0
        old = [s for s in range(min(sinks, first))] + list(range(first, h))
        live = [i for i in range(n) if trees is None or trees[b][i]]
        at = {i: h + (i if trees is None else len(trees[b][i]) - 1) for i in live}
        pos = torch.tensor([at[i] for i in live], dtype=torch.long, device=DEV)
        here = torch.tensor(live, dtype=torch.long, device=DEV)
        kc[b, :, h + here] = _exact_turned(st["k"][b, here], pos, c).transpose(0, 1)
        vc[b, :, h + here] = st["v"][b, here].double().transpose(0, 1)
        q = _exact_turned(st["q"][b, here], pos, c)
        old_t = torch.tensor(old, dtype=torch.long, device=DEV)
        slots = torch.cat([old_t, h + here])
        place = torch.cat([old_t, pos])  # the position of each slot's token
        off = place[None] > pos[:, None]
        if window:
            off |= (pos[:, None] - place[None] >= window) & (place[None] >= sinks)
        if trees is not None:
            kin = torch.zeros((n, n), dtype=torch.bool)
            for i in live:
                kin[i, trees[b][i]] = True
            off[:, len(old):] |= ~kin[live][:, live].to(DEV)
        for head in range(c["hq"]):
            g = head // (c["hq"] // c["hkv"])
            a = (q[:, head] @ kc[b, g, slots].T) / math.sqrt(c["d"])
            out[b, here, head] = torch.softmax(a.masked_fill(off, -math.inf), -1) @ vc[b, g, slots]
    return {"out": out, "k_cache": kc, "v_cache": vc}
