"""64-bit definitions of the operators on quantised layers, on the CPU, and seeded inputs for them."""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a step
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def pack(codes):
    """int8 [n, k] in [-8, 7] to two codes a byte, low nibble first."""
    n, k = codes.shape
    c = torch.nn.functional.pad(codes, (0, k & 1)).view(torch.uint8)
    return ((c[:, 0::2] & 15) | (c[:, 1::2] << 4)).contiguous()


def codes_of(rng, n, k, fmt, full_range=True):
    top = 7 if fmt == "int4" else 127
    low = -8 if fmt == "int4" else -128
    c = rng.integers(low if full_range else -top, top + 1, (n, k)).astype(np.int8)
    return torch.from_numpy(c)


def act64(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def strided(t, pad, device):
    """t on the device with `pad` elements between its rows (they hold NaN)."""
    buf = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=device)
    view = buf[:, :t.shape[1]]
    view.copy_(t)
    return view


def sum_error(terms_rms, depth):
    """Bound of the error of a binary32 sum of `depth` products whose root-sum-square is `terms_rms`: a rounding
    or truncation of at most 2^-23 of the running sum for each group of 8 products the matrix units add, the
    running sum of terms of random signs taken as at most 4 times the root-sum-square; and 2^-22 of each term
    where a binary32 operand goes in as two 11-bit halves."""
    return terms_rms * (4 * (depth / 8 + 8) * 2.0 ** -23 + 2.0 ** -20)
