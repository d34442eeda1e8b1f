"""Plain 64-bit statements of the operators of a decoder's 8-bit pass, on the CPU."""
from __future__ import annotations

import numpy as np
import torch

from decoder_util import e4m3_grid


def up(n, m):
    return -(-n // m)


def quantise(y: np.ndarray, block=32, block_rows=1):
    """[rows, cols] -> codes uint8, scale bytes uint8 [ceil(rows / block_rows), ceil(cols / block)], by the definition."""
    rows, cols = y.shape
    g = np.zeros((up(rows, block_rows) * block_rows, up(cols, block) * block))
    g[:rows, :cols] = y
    g = g.reshape(-1, block_rows, up(cols, block), block)
    fin = np.isfinite(g).all((1, 3), keepdims=True)                     # a block that is not finite is NaN as a whole
    mag = np.where(fin, np.abs(g), 0.0)
    amax = mag.max((1, 3), keepdims=True)
    k = np.full(amax.shape, -120)
    for e in range(-120, 120):                                          # smallest power with amax <= 448 * 2^k
        k = np.where(amax > 448.0 * 2.0 ** e, min(e + 1, 119), k)
    grid = e4m3_grid()
    mag = mag / np.exp2(k.astype(np.float64))
    hi = np.clip(np.searchsorted(grid, mag), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    above, below = grid[hi] - mag, mag - grid[lo]
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    code = np.where(mag >= grid[-1], 0x7E, code)
    code = np.where(fin, code | (np.signbit(g) * 0x80), 0x7F).astype(np.uint8)
    scale = np.where(fin, k + 127, 255).astype(np.uint8)
    return code.reshape(-1, g.shape[2] * block)[:rows, :cols].copy(), scale.reshape(up(rows, block_rows), -1).copy()


def values(codes: np.ndarray, scale: np.ndarray, block=32, block_rows=1) -> np.ndarray:
    rows, cols = codes.shape
    grid = np.append(e4m3_grid(), np.nan)
    v = grid[codes & 0x7F] * np.where(codes & 0x80, -1.0, 1.0)
    step = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return v * np.repeat(np.repeat(step, block_rows, 0)[:rows], block, 1)[:, :cols]


def rotated(x: torch.Tensor, weight, place, inv_freq, interleaved, eps):
    """x [n, heads, dim] (64 bits) normalised and rotated, and the sum of the two products' magnitudes for every element."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    half = len(inv_freq)
    pair = torch.arange(half)
    a, b = (2 * pair, 2 * pair + 1) if interleaved else (pair, pair + half)
    angle = place.double()[:, None, None] * inv_freq.double()
    c, s = angle.cos(), angle.sin()
    out, size = y.clone(), y.abs()
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
    return out, size


def scores(z: torch.Tensor, tokens, k):
    """logprob, entropy, rank, top, top_logprob of rows of 64-bit logits that are all in order; tokens may hold -1."""
    V = z.shape[1]
    d = z - z.amax(1, keepdim=True)                 # first: logits as large as 1e38 would swallow the logarithm of the sum
    logp = d - d.exp().sum(1, keepdim=True).log()
    entropy = -(torch.where(logp.isinf(), torch.zeros(()).double(), logp) * logp.exp()).sum(1)
    order = torch.sort(z + 0.0, dim=1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(1, order, torch.arange(V).expand_as(order))
    t = tokens.long().clamp_min(0)[:, None]
    none = tokens < 0
    lp, rank = logp.gather(1, t)[:, 0], place.gather(1, t)[:, 0]
    top = order[:, :k]
    top_lp = logp.gather(1, top)
    pad = max(0, k - V)
    top, top_lp = torch.nn.functional.pad(top, (0, pad), value=-1), torch.nn.functional.pad(top_lp, (0, pad), value=-float("inf"))
    return torch.where(none, torch.nan, lp), entropy, torch.where(none, -1, rank), top, top_lp
