"""Oracle of the hard quantiser with group scales and of products with its codes.  Test infrastructure: plain float64, written
out from the definitions; nothing here is shared with the CUDA path.

A group is ``group`` consecutive weights of a row (the last may be shorter); its scale is max|w| / max|c|, divided in float32 and
rounded to the type of the codebook; a weight gets the lowest index j among those with the smallest |w - s c_j|.  Codes are
4 bits, even columns in the low half of a byte, rows padded with zeros to 16 bytes.
"""
from __future__ import annotations

import numpy as np
import torch


def assign(W: torch.Tensor, C: torch.Tensor, group: int):
    """(indices [rows, cols] uint8, scales [rows, groups] of C's type, dequantised weights of W's type), CPU tensors."""
    rows, cols = W.shape
    w32, c32 = W.float().numpy(), C.float().numpy().reshape(-1)
    good = np.isfinite(c32)
    c_max = np.float32(np.abs(c32[good]).max()) if good.any() else np.float32(0)
    c64 = np.where(good, c32.astype(np.float64), np.nan)
    n = -(-cols // group)
    idx = np.zeros((rows, cols), np.uint8)
    scales = torch.zeros(rows, n, dtype=C.dtype)
    held = np.zeros((rows, n), np.float32)
    with np.errstate(all="ignore"):
        for g in range(n):
            w = w32[:, g * group:(g + 1) * group]
            s = torch.from_numpy(np.abs(w).max(1) / c_max if c_max > 0 else np.zeros(rows, np.float32)).to(C.dtype)
            scales[:, g] = s
            held[:, g] = s.float().numpy()
            d = np.abs(w.astype(np.float64)[:, :, None] - held[:, g].astype(np.float64)[:, None, None] * c64[None, None, :])
            d = np.where(np.isnan(d), np.inf, d)
            j = np.argmin(d, axis=2)
            j[~np.isfinite(held[:, g])] = 0
            j[held[:, g] == 0] = 0
            idx[:, g * group:(g + 1) * group] = j
        s_of = np.repeat(held, group, axis=1)[:, :cols]
        Wq = torch.from_numpy(s_of * np.where(good, c32, np.float32(np.nan))[idx]).to(W.dtype)
    return idx, scales, Wq


def pack(idx) -> np.ndarray:
    rows, cols = idx.shape
    full = np.zeros((rows, (cols + 31) // 32 * 32), np.uint8)
    full[:, :cols] = idx
    return (full[:, 0::2] | (full[:, 1::2] << 4)).astype(np.uint8)


def unpack(codes, cols: int) -> np.ndarray:
    codes = np.asarray(codes, np.uint8)
    out = np.empty((codes.shape[0], codes.shape[1] * 2), np.uint8)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out[:, :cols]


def weights(codes, C, scales, group: int, cols: int) -> np.ndarray:
    """The weights that the codes stand for, float64 [rows, cols]; a code past the codebook stands for 0."""
    c = np.zeros(16)
    flat = C.double().numpy().reshape(-1)
    c[:flat.size] = flat
    w = c[unpack(codes, cols)]
    if scales is not None:
        w = w * np.repeat(scales.double().numpy(), group, axis=1)[:, :cols]
    return w


def matmul(X: torch.Tensor, codes, C, scales, group: int):
    """(X W^T, |X| |W|^T): the product in float64, and the sum of its terms' sizes, which rounding errors are relative to."""
    w, x = weights(codes, C, scales, group, X.shape[1]), X.double().numpy()
    return x @ w.T, np.abs(x) @ np.abs(w).T
