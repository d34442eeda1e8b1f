"""Plain 64-bit statements of the decoder-side operators, and the inputs their tests share.

8-bit blocks are handled as numbers here: a value's code is found by searching e4m3's grid, not by a
type conversion."""
from __future__ import annotations

import numpy as np
import torch

BLOCK = 32


def e4m3_grid() -> np.ndarray:
    """Values of the codes 0x00 .. 0x7E (0x7F is NaN), ascending."""
    g = []
    for c in range(0x7F):
        e, m = c >> 3, c & 7
        g.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(g)


def quantise(x: np.ndarray):
    """[..., n] -> (codes uint8 [..., n], scale bytes [..., n / 32]) by the definition."""
    g = x.astype(np.float64).reshape(*x.shape[:-1], -1, BLOCK)
    fin = np.isfinite(g).all(-1, keepdims=True)      # a block that is not finite is NaN as a whole
    amax = np.where(fin, np.abs(g), 0.0).max(-1)
    k = np.full(amax.shape, -120)
    for e in range(-120, 120):                      # smallest power with amax <= 448 * 2^k
        k = np.where(amax > 448.0 * 2.0 ** e, min(e + 1, 119), k)
    grid = e4m3_grid()
    mag = np.where(fin, np.abs(g), 0.0) / 2.0 ** k[..., None].astype(np.float64)
    hi = np.clip(np.searchsorted(grid, mag), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(mag >= grid[-1], 0x7E, code)
    code = np.where(fin, code | (np.signbit(g) * 0x80), 0x7F)
    return code.astype(np.uint8).reshape(x.shape), np.where(fin[..., 0], k + 127, 255).astype(np.uint8)


def values(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    grid = np.append(e4m3_grid(), np.nan)
    v = grid[codes & 0x7F] * np.where(codes & 0x80, -1.0, 1.0)
    step = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v.reshape(*codes.shape[:-1], -1, BLOCK) * step[..., None]).reshape(codes.shape)


class Context:
    """A paged cache with the contexts of a batch in it, on the CPU in 64 bits and on the GPU as the
    library takes it.  Slots that hold no token are NaN; table entries past a context are far out of range."""

    def __init__(self, new, length, heads, dim, page, fmt="bf16", seed=0, layout="head", stale=float("nan"), fill=None):
        rng = np.random.default_rng(seed)
        self.new, self.length, self.heads, self.dim, self.page, self.fmt = list(new), list(length), heads, dim, page, fmt
        B = len(new)
        pages = [-(-max(l, 0) // page) for l in length]
        self.n_pages = max(1, sum(pages)) + 2
        width = max(1, max(pages))
        order = rng.permutation(self.n_pages)
        self.table = np.full((B, width), 1 << 29, np.int32)
        at = 0
        for b in range(B):
            self.table[b, :pages[b]] = order[at:at + pages[b]]
            at += pages[b]
        shape = (self.n_pages, heads, page, dim)
        self.host, self.dev = {}, {}
        for name in "kv":
            dense = [torch.from_numpy(rng.normal(0, 1, (max(l, 0), heads, dim))).bfloat16() for l in length]
            if fill is not None:
                dense = [fill(name, b, x) for b, x in enumerate(dense)]
            pool = torch.full(shape, stale, dtype=torch.bfloat16)
            for b in range(B):
                for j in range(pages[b]):
                    rows = dense[b][j * page:(j + 1) * page].transpose(0, 1)
                    pool[self.table[b, j], :, :rows.shape[1]] = rows
            if fmt == "e4m3":
                codes, scale = quantise(pool.float().numpy())
                dense = [torch.from_numpy(values(*quantise(x.float().numpy()))) if x.numel() else x.double() for x in dense]
                pool = torch.from_numpy(codes)
                self.dev[name + "_scale"] = torch.from_numpy(scale).cuda()
            if layout == "token":                  # [n_pages, page, heads, dim] seen as [n_pages, heads, page, dim]
                pool = pool.transpose(1, 2).contiguous().cuda().transpose(1, 2)
            elif layout == "padded":               # both pools in one allocation, rows padded
                wide = torch.zeros(self.n_pages, heads, page, dim + 16, dtype=pool.dtype)
                wide[..., :dim] = pool
                pool = wide.cuda()[..., :dim]
            else:
                pool = pool.cuda()
            self.host[name], self.dev[name] = [x.double() for x in dense], pool
        self.new_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.d_table = torch.from_numpy(self.table).cuda()
        self.d_new_start = torch.from_numpy(self.new_start).cuda()
        self.d_len = torch.tensor(list(length), dtype=torch.int32).cuda()

    def cache(self, E):
        return E.ead_kv_cache(self.dev["k"], self.dev["v"], self.dev.get("k_scale"), self.dev.get("v_scale"))

    def batch(self, E, **kw):
        return E.ead_kv_batch(self.d_table, self.d_new_start, self.d_len,
                              **{**dict(n_tokens=int(self.new_start[-1]), max_new=max(self.new), max_len=max(max(self.length), 0)), **kw})


def attention(ctx: Context, q: torch.Tensor, scale, window, sinks):
    """out, lse and the tolerances of both, in 64 bits on the CPU.

    Out: the probabilities are rounded to bf16 (8 significant bits, relative 2^-8 each) and so is the result; a logit is a
    32-bit sum of head_dim products (2^-24 each in the worst case, 2^-18 of the sum of magnitudes covers
    head_dim 128 and the few roundings around it) and its error enters every probability."""
    n, hq, dim = q.shape
    group = hq // ctx.heads
    out = torch.zeros(n, hq, dim, dtype=torch.float64)
    lse = torch.full((n, hq), -np.inf, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros(n, hq, dtype=torch.float64)
    t = 0
    for b, (m, l) in enumerate(zip(ctx.new, ctx.length)):
        if m and l > 0:
            k, v = (ctx.host[x][b].transpose(0, 1).repeat_interleave(group, 0) for x in "kv")     # [hq, l, dim]
            x = q[t:t + m].double().transpose(0, 1)
            z = scale * (x @ k.transpose(1, 2))
            pos = torch.arange(l - m, l)[:, None]
            key = torch.arange(l)[None]
            seen = key <= pos
            if window:
                seen = seen & ((key > pos - window) | (key < sinks))
            rough = scale * (x.abs() @ k.abs().transpose(1, 2))
            rough = torch.where(seen, rough, torch.zeros(())).amax(-1) * 2.0 ** -18
            z = torch.where(seen, z, torch.full((), -np.inf, dtype=torch.float64))
            e = torch.logsumexp(z, -1)
            p = torch.where(seen.any(-1)[None, :, None], torch.exp(z - e[..., None]), torch.zeros((), dtype=torch.float64))
            v = torch.nan_to_num(v) if not seen.all() else v
            o, w = p @ v, p @ v.abs()
            out[t:t + m], lse[t:t + m] = o.transpose(0, 1), e.transpose(0, 1)
            tol_o[t:t + m] = ((2.0 ** -8 * 1.02 + 2 * rough[..., None] + 2.0 ** -18) * w + 2.0 ** -8 * 1.02 * o.abs() + 1e-30).transpose(0, 1)
            tol_l[t:t + m] = (rough + 2.0 ** -20 * (1 + torch.nan_to_num(e, neginf=0.0).abs())).transpose(0, 1)
        t += m
    return out, lse, tol_o, tol_l
