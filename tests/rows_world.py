"""A cache of sessions for the tests of rows and 8-bit values, its slots on
the host in 64 bits, and the operators in 64 bits, written from their
definitions in memdecay.h (no code shared with the library)."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2607_10582_amd.cache import MemDecay, PagedCache

D = 128
BF16 = torch.bfloat16


def quantise(v):
    """Blocks [n][16][heads][d] (zeros where there is no token) -> the values
    that codes and scales stand for, float64, and the scales [n][heads]."""
    x = v.float()
    top = x.abs().amax((1, 3))
    scale = (top / 448.0).masked_fill(~torch.isfinite(top), math.nan)
    q = x / torch.where(scale > 0, scale, 1.0)[:, None, :, None]
    codes = torch.where((scale > 0)[:, None, :, None], q, 0.0).to(torch.float8_e4m3fn)
    return codes.double() * scale.double()[:, None, :, None], scale


def quantise_slots(v):
    """Slots [n][heads][d] -> what they read as in 8 bits."""
    n = v.shape[0]
    full = torch.zeros((-(-n // 16) * 16,) + tuple(v.shape[1:]), dtype=v.dtype)
    full[:n] = v
    return quantise(full.view(-1, 16, *v.shape[1:]))[0].flatten(0, 1)[:n]


def attend(q, k, v, seen):
    """q [G][d], k, v [n][d], seen [n] -> out [G][d], lse [G], and the mean
    distance of the values from the result, sum p |v - out| [G][d]."""
    k, v = k[seen].double(), v[seen].double()
    q = q.double()
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full((q.shape[0],), -math.inf, dtype=torch.float64), torch.zeros_like(q)
    x = q @ k.T / math.sqrt(D)
    top = x.max(1, keepdim=True).values
    w = torch.exp(x - top)
    z = w.sum(1, keepdim=True)
    out = w @ v / z
    dev = torch.stack([(p[:, None] * (v - o).abs()).sum(0) for p, o in zip(w / z, out)])
    return out, (top + torch.log(z))[:, 0], dev


def visible(live, own, window, sinks):
    """The slots that the row at slot `own` sees."""
    j = np.arange(len(live))
    seen = np.asarray(live) & (j <= own)
    if window:
        seen &= (own - j < window) | (j < sinks)
    return torch.as_tensor(seen)


class World:
    """Sessions of `lens` tokens; every slot without one holds NaN."""

    def __init__(self, L, Hq, Hkv, P, lens, seed=1, coded=True, aligned=False, quant=0.0, extra=4, spare=2, scale=1.0, stream=None,
                 fill=True, quant_threshold=None, **kw):
        self.L, self.Hq, self.Hkv, self.P, self.S, self.G = L, Hq, Hkv, P, len(lens), Hq // Hkv
        self.coded, self.aligned = coded, aligned
        g = self.g = torch.Generator().manual_seed(seed)
        rng = self.rng = np.random.default_rng(seed)
        self.regions = [np.repeat(rng.integers(0, 7, n // 5 + 1), 5)[:n].astype(np.uint8) for n in lens]
        pages = [PagedCache.pages_for(r, P, aligned) for r in self.regions]
        NP = sum(pages) + spare * self.S + 1
        c = self.cache = PagedCache(L=L, Hq=Hq, Hkv=Hkv, d=D, P=P, S=self.S, max_pages=max(pages) + extra, n_phys=NP,
                                    values="e4m3" if coded else True, **kw)
        self.dev = c.device
        c.k_pool.fill_(math.nan)
        if coded:
            c.v_codes.fill_(0x7F)   # NaN
            c.v_scale.fill_(math.nan)
            c.v_open.fill_(math.nan)
        else:
            c.v_pool.fill_(math.nan)
        ids = rng.permutation(NP)
        self.ids, self.slots, self.live, self.k, self.v, self.v16 = [], [], [], [], [], []
        at = 0
        for s, n in enumerate(lens):
            mine = ids[at:at + pages[s]]
            at += pages[s]
            self.ids.append(mine)
            pos = PagedCache.positions(self.regions[s], P, aligned)
            slots = int(pos[-1]) + 1 if n else 0
            live = np.zeros(slots, bool)
            live[pos] = True
            k, v = (torch.zeros((slots, L, Hkv, D)) for _ in range(2))
            k[pos] = (torch.randn((n, L, Hkv, D), generator=g) * scale).to(BF16).float()
            v[pos] = torch.randn((n, L, Hkv, D), generator=g).to(BF16).float()
            self.slots.append(slots)
            self.live.append(live)
            self.k.append(k.double())
            self.v16.append(v)
            self.v.append(quantise_slots(v.flatten(1, 2)).view(slots, L, Hkv, D) if coded else v.double())
            if not fill:
                c.place_session(s, self.regions[s], mine, budget=n, clock=n, region_aligned=aligned)
            elif n:
                c.load_session(s, k[pos].to(BF16), self.regions[s], mine, budget=n, clock=n, region_aligned=aligned)
                c.load_values(s, v[pos].to(BF16), self.regions[s] if aligned else None)
                self._poison(s, live, pages[s])
                if quant > 0:
                    self._codes(s, pages[s], quant)
        c.set_free_pages(ids[at:])
        ones = torch.ones((self.S, 7))
        threshold = (0.3 if quant > 0 else 0.0) if quant_threshold is None else quant_threshold
        self.md = MemDecay(c, ones, ones * 0.01, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0, region_aligned=aligned,
                           quant_threshold=threshold, stream=stream)

    def _poison(self, s, live, pages):
        """NaN in the slots without a token."""
        c, P = self.cache, self.P
        own = torch.as_tensor(self.ids[s], device=self.dev)
        dead = np.ones(pages * P, bool)
        dead[:len(live)] = ~live
        at = torch.as_tensor(np.flatnonzero(dead), device=self.dev)
        x = PagedCache.from_pool_layout(c.k_pool[own]).contiguous()
        x.view(-1, self.L, self.Hkv, D)[at] = math.nan
        c.k_pool[own] = PagedCache.to_pool_layout(x)
        if not self.coded:
            x = PagedCache.from_value_layout(c.v_pool[own]).contiguous()
            x.view(-1, self.L, self.Hkv, D)[at] = math.nan
            c.v_pool[own] = PagedCache.to_value_layout(x)
            return
        x = c.v_codes[own].permute(0, 3, 5, 8, 1, 2, 4, 7, 6).contiguous()      # [m][P/16][4][4][L][Hkv][..]
        x.view(-1, *x.shape[4:])[at] = 0x7F
        c.v_codes[own] = x.permute(0, 4, 5, 1, 6, 2, 8, 7, 3)
        empty = dead.reshape(-1, 16).all(1).reshape(pages, P // 16)
        sc = c.v_scale[own].permute(0, 3, 1, 2).contiguous()
        sc[torch.as_tensor(empty, device=self.dev)] = math.nan
        c.v_scale[own] = sc.permute(0, 2, 3, 1)

    def _codes(self, s, pages, share):
        """Some full pages' keys become codes and scales."""
        c, P = self.cache, self.P
        for o in range(pages - 1):
            if self.rng.random() > share:
                continue
            x = self.k[s][o * P:(o + 1) * P].float().view(P // 16, 16, self.L * self.Hkv, D)
            back, scale = quantise(x)
            self.k[s][o * P:(o + 1) * P] = back.view(P, self.L, self.Hkv, D)
            q = (x / torch.where(scale > 0, scale, 1.0)[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            raw = torch.full((P // 16, self.L * self.Hkv, 4096), 0xFF, dtype=torch.uint8)
            e = torch.arange(D)
            for t in range(16):
                raw[..., 1024 * (e // 64) + 16 * (t + 16 * ((e // 8) % 4)) + 8 * ((e // 32) % 2) + e % 8] = q[:, t]
            raw[..., 2048:2064] = scale.contiguous().view(-1, 1).repeat(1, 4).view(torch.uint8).view(P // 16, -1, 16)
            page = int(self.ids[s][o])
            pool = c.k_pool.view(torch.uint8).view(c.n_phys, self.L, self.Hkv, P // 16, 4096)
            pool[page] = raw.view(P // 16, self.L, self.Hkv, 4096).permute(1, 2, 0, 3).to(self.dev)
            c.page_format[page] = 1

    def normal(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.g).to(dtype).to(self.dev)

    def i32(self, x):
        return torch.as_tensor(np.asarray(x, dtype=np.int32), device=self.dev)

    def rows(self, counts, first=None):
        """row_start and row_slot of `counts` rows of each session, its last
        ones or those from slot first[s] on (holes left out)."""
        start = np.concatenate([[0], np.cumsum(counts)])
        slot = []
        for s, n in enumerate(counts):
            at = np.flatnonzero(self.live[s])
            at = at[len(at) - n:] if first is None else at[np.searchsorted(at, first[s]):][:n]
            assert len(at) == n
            slot += at.tolist()
        return self.i32(start), self.i32(slot), start, np.array(slot, dtype=int)


def attention_bound(q, k, v, seen, dev, ref, rl, rounded, out_type):
    """Tolerances of one head group's outputs and log-sums.

    A logit is 3 * 128 exact products (rounded: 128) summed in float32: at most
    384 2^-24 sum |q_e k_e| / sqrt(d) off; a weight follows it twice (its own
    and the sum's), the exponential, the sums and the scales take 2^-20, three
    bf16 terms 2^-26.  A weight that is rounded to bf16 moves by up to 2^-8 of
    itself, and so does its share in the sum: the result by up to 2^-8 /
    (1 - 2^-8) of the mean distance of the values from it.  A bf16 output is
    rounded by up to 2^-8 of itself."""
    off = 0.0
    top = 0.0
    if bool(seen.any()):
        off = float((q.double().abs() @ k[seen].double().abs().T).max()) / math.sqrt(D) * 384 * 2.0 ** -24
        top = float(v[seen].abs().max())
    tol = torch.full_like(ref, (2 * off + 2.0 ** -26 + 2.0 ** -20) * top)
    if rounded:
        tol = tol + dev * (2.0 ** -8 / (1 - 2.0 ** -8))
    if out_type == BF16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)
    return tol, off + 2.0 ** -20 * (1 + torch.where(torch.isfinite(rl), rl.abs(), 0.0))
