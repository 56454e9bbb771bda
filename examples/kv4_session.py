"""A conversation through the attention halves of a few decoder blocks with their KV caches held in 4 bits.

Random W4BF16 weights.  The prompt goes through in chunks (kv4_prefill_kv, one workspace for all layers), then
tokens are decoded one by one from a CUDA graph (kv4_decode between the two GEMVs of a block), four drafted tokens
are verified in one pass, and the caches are read back as bf16 (kv4_read).  The same prompt and tokens with
bf16 caches tell what the 4 bits cost in accuracy.

  python examples/kv4_session.py [--layers 4] [--hidden 4096] [--heads 32] [--kv-heads 8] [--head-dim 128]
                                 [--prompt 6000] [--chunk 1024] [--steps 32]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

EPS = 1e-5


def weights(rows, cols, gen):
    """The tile stream of a random [rows, cols] matrix of deviation about 1 / sqrt(cols)."""
    import numpy as np
    import torch

    from paper_2607_15865_gb300.w4 import pack_codes, pack_tiles
    codes = gen.integers(0, 16, (rows, cols), dtype=np.uint8)
    zeros = gen.integers(7, 9, (rows, cols // 128), dtype=np.uint8)
    scale = np.float32(1.0 / (4.6 * np.sqrt(cols)))
    scales = np.full((rows, cols // 128), np.array([scale]).view(np.uint32)[0] >> 16, np.uint16)
    return torch.from_numpy(pack_tiles(pack_codes(codes), scales, zeros)).cuda()


def norm(x):
    import torch
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + EPS)).to(torch.bfloat16)


class Model:
    """Attention halves of decoder blocks; `caches` are 4-bit ones or (k, v) pairs of bf16 tensors."""

    def __init__(self, args, attn, gen):
        import torch
        self.a, self.attn = args, attn
        self.qd, self.kd = args.heads * args.head_dim, args.kv_heads * args.head_dim
        self.wqkv = [weights(self.qd + 2 * self.kd, args.hidden, gen) for _ in range(args.layers)]
        self.wo = [weights(args.hidden, self.qd, gen) for _ in range(args.layers)]
        self.gamma = torch.ones(args.hidden, dtype=torch.bfloat16, device="cuda")

    def _split(self, qkv, n):
        a = self.a
        q, k, v = qkv.split([self.qd, self.kd, self.kd], -1)
        return (q.reshape(1, n, a.heads, a.head_dim).contiguous(), k.reshape(1, n, a.kv_heads, a.head_dim).contiguous(),
                v.reshape(1, n, a.kv_heads, a.head_dim).contiguous())

    def chunk(self, x, hist, caches, workspace=None):
        """x [n, hidden] at positions hist .. -> the blocks' output."""
        from paper_2607_15865_gb300.w4 import w4bf16_gemm
        for i, cache in enumerate(caches):
            q, k, v = self._split(w4bf16_gemm(self.wqkv[i], norm(x), self.qd + 2 * self.kd), x.shape[0])
            if isinstance(cache, tuple):
                o = self.attn.prefill_kv(q, k, v, hist, *cache)
            else:
                o = self.attn.kv4_prefill_kv(q, k, v, hist, cache, workspace)
            x = x + w4bf16_gemm(self.wo[i], o.view(x.shape[0], self.qd), self.a.hidden)
        return x

    def tokens(self, x, lens, caches):
        """x [n, hidden], n <= 8 new tokens at positions lens[0] .., through the GEMVs and the decode."""
        from paper_2607_15865_gb300.w4 import w4bf16_gemv_fused
        n, a = x.shape[0], self.a
        for i, cache in enumerate(caches):
            q, k, v = w4bf16_gemv_fused(self.wqkv[i], x, self.qd + 2 * self.kd, self.gamma, EPS,
                                        split=(self.qd, self.qd + self.kd))
            q, k, v = q.view(1, n, a.heads, a.head_dim), k.view(1, n, a.kv_heads, a.head_dim), v.view(1, n, a.kv_heads, a.head_dim)
            if isinstance(cache, tuple):
                o = self.attn.decode_multi(q, k, v, lens, *cache)
            else:
                o = self.attn.kv4_decode(q, k, v, lens, cache)
            x = w4bf16_gemv_fused(self.wo[i], o.view(n, self.qd), a.hidden, residual=x)
        return x


def session(model, caches, prompt, drafts, workspace=None):
    """The hidden states of the prompt's last chunk, of each decoded token and of the drafts; us per step."""
    import torch
    a = model.a
    out, hist = None, 0
    for c in prompt.split(a.chunk):
        out = model.chunk(c, hist, caches, workspace)
        hist += c.shape[0]
    states = [out]
    lens = torch.tensor([hist], dtype=torch.int32, device="cuda")
    x = norm(out[-1:]).clone()
    y = model.tokens(x, lens, caches)  # rewrites slot `hist` when the graph runs it again
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = model.tokens(x, lens, caches)
        x.copy_(norm(y))
        lens += 1
    e0, e1 = torch.cuda.Event(True), torch.cuda.Event(True)
    e0.record()
    for _ in range(a.steps):
        g.replay()
        states.append(y.clone())
    e1.record()
    states.append(model.tokens(drafts, lens, caches))
    torch.cuda.synchronize()
    if model.attn.device_error():
        raise RuntimeError("a kernel reported an error")
    return states, e0.elapsed_time(e1) * 1e3 / max(a.steps, 1)


def main(argv=None):
    import numpy as np
    import torch

    from paper_2607_15865_gb300.attention import Attention
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("head-dim", 128),
                        ("prompt", 6000), ("chunk", 1024), ("steps", 32)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    total = a.prompt + a.steps + 4
    attn = Attention(1, a.heads, a.kv_heads, a.head_dim, total, 5.0e5)
    gen = np.random.default_rng(0)
    model = Model(a, attn, gen)
    torch.manual_seed(0)
    prompt, drafts = (torch.randn(n, a.hidden, device="cuda").to(torch.bfloat16) for n in (a.prompt, 4))
    packed = [attn.kv4_cache() for _ in range(a.layers)]
    plain = [tuple(torch.zeros(1, a.kv_heads, total, a.head_dim, dtype=torch.bfloat16, device="cuda") for _ in "kv")
             for _ in range(a.layers)]
    workspace = torch.empty(attn.kv4_workspace(a.prompt), dtype=torch.uint8, device="cuda")
    s4, us4 = session(model, packed, prompt, drafts, workspace)
    s16, us16 = session(model, plain, prompt, drafts)
    size = sum(t.numel() * t.element_size() for c in packed for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales))
    size16 = sum(t.numel() * 2 for c in plain for t in c)
    rel = lambda x, y: float((x.float() - y.float()).norm() / y.float().norm())  # noqa: E731
    # the first layer's keys and values do not depend on the caches before, but for those of the decoded tokens: the
    # first of them comes of the prompt's last state
    k, v = attn.kv4_read(packed[0], 0, a.prompt + 1)
    slots, first = slice(0, a.prompt), slice(a.prompt, a.prompt + 1)
    result = {"bytes": size, "bytes_bf16": size16, "us_per_token": us4, "us_per_token_bf16": us16,
              "prompt": rel(s4[0], s16[0]), "k": rel(k[:, :, slots], plain[0][0][:, :, slots]),
              "v": rel(v[:, :, slots], plain[0][1][:, :, slots]), "token": rel(s4[1], s16[1]), "drafts": rel(s4[-1], s16[-1]),
              "token_k": rel(k[:, :, first], plain[0][0][:, :, first]), "token_v": rel(v[:, :, first], plain[0][1][:, :, first])}
    print(f"caches: {size / 1e6:.1f} MB in 4 bits, {size16 / 1e6:.1f} MB in bf16")
    print(f"a decoded token: {us4:.1f} us through {a.layers} blocks, {us16:.1f} us with bf16 caches")
    print(f"first layer's cache against bf16: k {result['k']:.3f}, v {result['v']:.3f} (relative)")
    print(f"hidden states against bf16: {result['prompt']:.4f} of the prompt's last chunk, {result['token']:.4f} of the first "
          f"decoded token, {result['drafts']:.4f} of the drafted ones (relative)")
    return result


if __name__ == "__main__":
    main()
