"""The 4-bit KV cache (attn_kv4 of include/attn.h): the tensors of one layer's cache.

The D values of a slot are held in groups of 32 as 4-bit codes c with a scale s and a zero
point z, a value being (c - z) s, exactly a bf16; 4.5 bits per value.  Attention writes it
(kv4_append), reads it back (kv4_read) and attends over it (kv4_decode, kv4_prefill_kv).
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib

GROUP = 32


class Kv4Cache:
    """The four tensors of a cache of max_len slots, Lp = attn_kv4_slots(max_len):
    k_codes, v_codes uint8 [B, Hkv, Lp, D / 2]; k_scales, v_scales int16 (or uint16, bfloat16) bit patterns
    [B, Hkv, Lp, D / 32], all on one device.  The tensors stay the caller's and are updated in place; the attributes
    that hold them cannot be set, as the calls go by their addresses: other tensors are another cache."""

    k_codes = property(lambda self: self._tensors[0])
    k_scales = property(lambda self: self._tensors[1])
    v_codes = property(lambda self: self._tensors[2])
    v_scales = property(lambda self: self._tensors[3])

    def __init__(self, max_len: int, k_codes, k_scales, v_codes, v_scales):
        slots = _lib.load().attn_kv4_slots(int(max_len))
        for t, name in ((k_codes, "k_codes"), (v_codes, "v_codes"), (k_scales, "k_scales"), (v_scales, "v_scales")):
            codes = name.endswith("codes")
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"{name} must be a CUDA tensor")
            if t.dtype not in ((torch.uint8,) if codes else (torch.int16, torch.uint16, torch.bfloat16)):
                raise TypeError(f"{name} must hold {'uint8 codes' if codes else '16-bit scales'}")
            if t.dim() != 4 or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous tensor of 4 dimensions")
            if t.device != k_codes.device:
                raise ValueError(f"{name} is on {t.device}, k_codes on {k_codes.device}")
        B, H, Lp, half = k_codes.shape
        want = {"codes": (B, H, slots, half), "scales": (B, H, slots, 2 * half // GROUP)}
        for t, name in ((k_codes, "k_codes"), (v_codes, "v_codes"), (k_scales, "k_scales"), (v_scales, "v_scales")):
            shape = want[name[2:]]
            if slots == 0 or half not in (32, 64) or tuple(t.shape) != shape:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape} (head_dim 64 or 128)")
        self.max_len = int(max_len)
        self._tensors = (k_codes, k_scales, v_codes, v_scales)
        self.shape = (B, H, self.max_len, 2 * half)
        self.struct = _lib.AttnKv4(*(t.data_ptr() for t in self._tensors))
        self.ref = ctypes.pointer(self.struct)

    @classmethod
    def empty(cls, batch: int, n_kv_heads: int, max_len: int, head_dim: int, device="cuda") -> "Kv4Cache":
        """A zeroed cache (every slot reads as 0)."""
        slots = _lib.load().attn_kv4_slots(int(max_len))
        codes = [torch.zeros((batch, n_kv_heads, slots, head_dim // 2), dtype=torch.uint8, device=device) for _ in "kv"]
        scales = [torch.zeros((batch, n_kv_heads, slots, head_dim // GROUP), dtype=torch.int16, device=device)
                  for _ in "kv"]
        return cls(max_len, codes[0], scales[0], codes[1], scales[1])
