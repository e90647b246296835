"""Plain implementation (NumPy, torch in 64 bits) of what include/tpq.h says about 4-bit weights, products with them, the gated block and answers."""
from __future__ import annotations

import math

import numpy as np
import torch

TILE = 128


def quantise(w: np.ndarray, group: int):
    """w [n][K] float64 (BF16 values) -> codes int [n][K], step bytes [n][groups], factors float32 [n]."""
    n, K = w.shape
    G = -(-K // group)
    pad = np.zeros((n, G * group))
    pad[:, :K] = w
    a = np.abs(pad).reshape(n, G, group).max(2)
    bad = ~(a.max(1) < 2.0 ** 120)
    a = np.where(bad[:, None], 0.0, a)
    b = np.where(a > 0, a, 1.0) * 2 / 15
    e = np.floor(np.log2(b)).astype(int)                       # (2a/15 is next to no power of two but those it equals)
    e = e + (b >= 2.0 ** (e + 1)) - (b < 2.0 ** e.astype(float))
    m = np.ceil(b.astype(np.float32) / 2.0 ** (e - 4.0))       # 16 .. 32
    e, m = np.where(m == 32, e + 1, e), np.where(m == 32, 16, m).astype(int)
    e = np.where(a > 0, e, -10 ** 6)
    E = np.maximum(e.max(1), -87)
    small = e < E[:, None] - 15
    e, m = np.where(small, E[:, None] - 15, e), np.where(small, 16, m)
    byte = ((e - E[:, None] + 15) * 16 + m - 16).astype(np.uint8)
    step = m * 2.0 ** (e - 4.0)
    factor = np.where(bad, np.nan, 2.0 ** (E - 7.0)).astype(np.float32)
    x = np.where(bad[:, None], 0.0, np.nan_to_num(w)) / np.repeat(step, group, 1)[:, :K]
    return np.clip(np.rint(x), -8, 7).astype(int), np.where(bad[:, None], 0, byte), factor


def values(codes, byte, factor, group):
    """float64 [n][K]: step * code."""
    step = factor[:, None].astype(float) * 2.0 ** ((byte >> 4).astype(float) - 8) * (1 + (byte & 15) / 16)
    return np.repeat(step, group, 1)[:, : codes.shape[1]] * codes


def pack(codes, byte, factor, group) -> np.ndarray:
    """The bytes of the layout."""
    n, K = codes.shape
    tiles, blocks, groups = -(-n // TILE), -(-K // TILE), TILE // group
    u = np.full((tiles * TILE, blocks * TILE), 8, np.uint32)
    u[:n, :K] = codes + 8
    step = np.zeros((tiles * TILE, blocks * groups), np.uint8)
    step[:n, : byte.shape[1]] = byte
    u = u.reshape(tiles, TILE, blocks, 4, 4, 4, 2)             # tile, output, block, 16-byte piece, word, pair, one of the pair
    i = np.arange(4, dtype=np.uint32)
    word = ((u[..., 0] << (4 * i)) | (u[..., 1] << (16 + 4 * i))).sum(-1).astype(np.uint32)
    codes_at = np.ascontiguousarray(word.transpose(0, 2, 3, 1, 4)).view(np.uint8).reshape(tiles, blocks, -1)     # tile, block, piece, output, word
    steps_at = step.reshape(tiles, TILE, blocks, groups).transpose(0, 2, 3, 1).reshape(tiles, blocks, -1)
    f = np.full(tiles * TILE, 2.0 ** -94, np.float32)          # (rows of nobody: the factor of a row of zeros)
    f[:n] = factor
    return np.concatenate([np.concatenate([codes_at, steps_at], 2).reshape(-1), f.view(np.uint8)])


def act(g: torch.Tensor, kind: int) -> torch.Tensor:
    if kind == 0:
        return g * torch.sigmoid(g)
    if kind == 1:
        return torch.nn.functional.gelu(g, approximate="tanh")
    return 0.5 * g * torch.special.erfc(-g / math.sqrt(2))       # (1 + erf z loses all digits below z = -6, in 64 bits too)


def gated(x, wg, wu, kind):
    """(out, bound of the error of binary32 sums and of the activation's slope) in 64 bits; sums of K products of binary32: K 2^-24 sum |x w|."""
    K = x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    dg, du = (K * 2.0 ** -24 * (x.abs() @ w.abs().T) for w in (wg, wu))
    a = act(g, kind)
    # |act'| <= 1.13 for all three; the activation itself: a few roundings of binary32
    da = 1.13 * dg + 16 * 2.0 ** -24 * (a.abs() + g.abs() * 2.0 ** -8)
    return a * u, da * (u.abs() + du) + a.abs() * du


def answers(x: torch.Tensor, tokens, n_top):
    """x [T][V] float64 on the CPU -> logprob, entropy, top, top_logprob."""
    T, V = x.shape
    m = x.amax(1, keepdim=True)
    none = torch.isneginf(m[:, 0])
    d = torch.where(none[:, None], x, x - torch.where(none, torch.zeros_like(m[:, 0]), m[:, 0])[:, None])   # (x - ln sum e^x loses the logarithm beside lowest numbers)
    logp = torch.where(none[:, None], x, d - torch.log(d.exp().sum(1, keepdim=True)))
    logp = torch.where(torch.isneginf(logp.float()), -math.inf, logp)   # (what binary32 cannot hold)
    p = logp.exp()
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(logp)).sum(1)
    at = torch.as_tensor(tokens).long()
    logprob = torch.where(at < 0, torch.zeros(T, dtype=x.dtype), logp[torch.arange(T), at.clamp(0, V - 1)])
    order = torch.argsort(x, dim=1, descending=True, stable=True)[:, :n_top]
    return logprob, entropy, order.to(torch.int32), logp.gather(1, order)
