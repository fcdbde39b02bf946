"""Tables of cosines and sines for the position rotation of bros_qkv_append."""

from __future__ import annotations

import torch


def rope_table(num_positions: int, rotary_dim: int = 128, base: float = 10000.0, inv_freq=None, device="cuda"):
    """float32 [num_positions][rotary_dim]: for position p and pair i the cosine of
    p * f_i at i and its sine at rotary_dim / 2 + i, with f_i = base^(-2 i / rotary_dim)
    or inv_freq[i]. Angles are formed in 64 bits: at position 100000 an angle of
    32 bits is off by 0.004."""
    if rotary_dim <= 0 or rotary_dim % 2:
        raise ValueError(f"rotary_dim {rotary_dim} must be positive and even")
    half = rotary_dim // 2
    if inv_freq is None:
        freq = base ** (-torch.arange(half, dtype=torch.float64) / half)
    else:
        freq = torch.as_tensor(inv_freq, dtype=torch.float64).cpu()
        if freq.shape != (half,):
            raise ValueError(f"inv_freq must hold {half} values")
    angles = torch.arange(num_positions, dtype=torch.float64)[:, None] * freq[None, :]
    return torch.cat([angles.cos(), angles.sin()], dim=1).float().to(device)
