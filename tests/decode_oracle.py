"""The decode operators in 64 bits, written from their definitions in
memdecay.h (test infrastructure only): plain loops over sessions and heads,
no code shared with the library."""
from __future__ import annotations

import math

import numpy as np
import torch

MIN_EXP, MAX_EXP = -100, 100


def norm_rope(x, weight, eps, position, inv_freq, interleaved):
    """Heads x [n][heads][d] (float64) -> the same, normalised and turned."""
    x = x.double().clone()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    half = 0 if inv_freq is None else inv_freq.numel()
    y = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        ang = position.double() * float(inv_freq[i])
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attend(q, k, v):
    """One head group: q [G][d], k, v [n][d] -> (out [G][d], lse [G])."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    x = q @ k.T / math.sqrt(q.shape[1])
    top = x.max(1, keepdim=True).values
    w = torch.exp(x - top)
    z = w.sum(1, keepdim=True)
    return w @ v / z, (top + torch.log(z))[:, 0]


def step_exp(amax: float) -> int:
    """The least e in [MIN_EXP, MAX_EXP] with amax <= 127 * 2^e."""
    e = MIN_EXP
    while e < MAX_EXP and amax > 127.0 * 2.0 ** e:
        e += 1
    return e


def bounds(k):
    """Keys [n][d] of a page -> (lo [d], hi [d], e), whole multiples of 2^e."""
    k = np.asarray(k, np.float64)
    e = step_exp(float(np.abs(k).max()))
    lo = np.clip(np.floor(k.min(0) / 2.0 ** e), -127, 127)
    hi = np.clip(np.ceil(k.max(0) / 2.0 ** e), -127, 127)
    return lo.astype(np.int64), hi.astype(np.int64), e


def block_score(q, lo, hi, e):
    """Largest bound over the group's query heads q [G][d]."""
    best = -math.inf
    for x in np.asarray(q, np.float64):
        x = np.where(np.isnan(x), 0.0, x)
        f = step_exp(float(np.abs(x).max()))
        c = np.clip(np.rint(np.clip(x, -3e38, 3e38) / 2.0 ** f), -127, 127).astype(np.int64)
        best = max(best, float(int((np.where(c > 0, c * hi, c * lo)).sum())) * 2.0 ** (e + f))
    return best


def select(scores, most, first, last):
    """Logical pages, ascending, of a session whose pages score ``scores``."""
    n = len(scores)
    if n <= most:
        return list(range(n))
    forced = [p for p in range(n) if p < first or p >= n - last]
    rest = sorted((p for p in range(n) if p not in set(forced)), key=lambda p: (-scores[p], p))
    return sorted(forced + rest[:most - len(forced)])
