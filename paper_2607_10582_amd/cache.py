"""Caller-side buffers and a thin driver for the MemDecay C ABI.

``PagedCache`` owns (through PyTorch) every device buffer of the library's
cache view: the paged bf16 key pool, the per-slot side arrays (region,
insertion step, refresh clock, importance), the page tables, the per-session
counters and the free list.  ``MemDecay`` binds a cache to a library handle
and calls the entry points in order.  PyTorch only allocates memory, places
the initial prompt into the pool (the decode engine's prefill, not part of
the retention step) and provides the stream; every step of the path runs in
the library's kernels.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B


class PagedCache:
    """Device buffers of one batch of sessions (layouts as in memdecay.h)."""

    def __init__(self, *, L: int, Hq: int, Hkv: int, d: int, P: int, S: int,
                 max_pages: int, n_phys: int, device="cuda", offload_pages: int = 0, values=False,
                 bounds: bool = False):
        # values: a pool of values beside the keys (MemDecay.attend), True for
        # bf16 ones, "e4m3" for 8-bit codes with a scale per 16 tokens and KV
        # head; bounds: 8-bit bounds of each page's keys (MemDecay.select_blocks)
        if values is None or values in (False, True):
            values = bool(values)
        elif values != "e4m3":
            raise ValueError('values are True (bf16), "e4m3" or False')
        self.L, self.Hq, self.Hkv, self.d, self.P = L, Hq, Hkv, d, P
        self.S, self.max_pages, self.n_phys = S, max_pages, n_phys
        self.device = torch.device(device)
        dev = self.device
        i32 = dict(dtype=torch.int32, device=dev)
        # Slots past a session's token count are never used, so the pool is
        # left uninitialised.
        self.k_pool = torch.empty((n_phys, L, Hkv, P // 16, d // 8, 16, 8), dtype=torch.bfloat16, device=dev)
        self.region = torch.zeros((n_phys, P), dtype=torch.uint8, device=dev)
        self.t_ins = torch.zeros((n_phys, P), **i32)
        self.t_ref = torch.zeros((n_phys, P), **i32)
        self.importance = torch.zeros((n_phys, P), dtype=torch.float32, device=dev)
        self.page_table = torch.full((S, max_pages), -1, **i32)
        self.page_serial = torch.full((S, max_pages), -1, **i32)
        self.n_pages = torch.zeros(S, **i32)
        self.n_tokens = torch.zeros(S, **i32)
        self.n_live = torch.zeros(S, **i32)   # tokens without holes (region-aligned pages)
        self.page_format = torch.zeros(n_phys, dtype=torch.uint8, device=dev)   # 1: quantised page
        self.clock = torch.zeros(S, **i32)
        self.next_serial = torch.zeros(S, **i32)
        self.budget = torch.zeros(S, **i32)
        self.free_list = torch.zeros(n_phys, **i32)
        self.free_count = torch.zeros(1, **i32)
        # pages past a session's table are never read, so the pools are left
        # uninitialised
        self.v_pool = torch.empty((n_phys, L, Hkv, P // 16, d // 32, 4, 16, 2, 4), dtype=torch.bfloat16,
                                  device=dev) if values is True else None
        coded = values == "e4m3"
        self.v_codes = torch.empty((n_phys, L, Hkv, P // 16, d // 64, 4, 16, 4, 4), dtype=torch.uint8,
                                   device=dev) if coded else None
        self.v_scale = torch.empty((n_phys, L, Hkv, P // 16), dtype=torch.float32, device=dev) if coded else None
        # the block that each session wrote last, in bf16, the one it wrote before
        # that, and which these are
        self._v_open, self.v_before = (torch.zeros((S, L, Hkv, 16, d), dtype=torch.bfloat16, device=dev) if coded else None
                                       for _ in range(2))
        self.v_held = torch.full((S, L, Hkv, 4), -1, **i32) if coded else None
        self.key_bounds = torch.empty((n_phys, L, Hkv, 2, d), dtype=torch.int8, device=dev) if bounds else None
        self.bound_exp = torch.empty((n_phys, L, Hkv), dtype=torch.int8, device=dev) if bounds else None
        # offload tier: offload_pages host-memory pages per session, their
        # keys in pinned host memory (hipHostMalloc underneath), their
        # per-token state on the device
        self.offload_pages = H = int(offload_pages)
        if H > 0:
            self.host_keys = torch.zeros((S, H, L * Hkv * P * d), dtype=torch.bfloat16, pin_memory=True)
            self.off_count = torch.zeros(S, **i32)
            self.off_serial = torch.full((S, H), -1, **i32)
            self.off_slot = torch.full((S, H), -1, **i32)
            self.off_region = torch.zeros((S, H, P), dtype=torch.uint8, device=dev)
            self.off_t_ins = torch.zeros((S, H, P), **i32)
            self.off_t_ref = torch.zeros((S, H, P), **i32)
            self.off_importance = torch.zeros((S, H, P), dtype=torch.float32, device=dev)
            self.off_format = torch.zeros((S, H), dtype=torch.uint8, device=dev)
            self.off_score = torch.zeros((S, H), dtype=torch.float32, device=dev)
            self.off_abar = torch.zeros((S, H, P), dtype=torch.float32, device=dev)

    @property
    def v_open(self) -> Optional[torch.Tensor]:
        return self._v_open

    @v_open.setter
    def v_open(self, blocks: torch.Tensor):
        # what a caller's own blocks hold is not known: they are taken for the
        # block that a session's rows go on in (memdecay.h)
        self._v_open = blocks
        self.v_before = self.v_held = None

    OFFLOAD_BUFFERS = ("host_keys", "off_count", "off_serial", "off_slot", "off_region", "off_t_ins",
                       "off_t_ref", "off_importance", "off_format", "off_score", "off_abar")

    def view(self) -> B.md_cache_view:
        v = B.md_cache_view()
        names = ["k_pool", "region", "t_ins", "t_ref", "importance", "page_table",
                 "page_serial", "n_pages", "n_tokens", "clock", "next_serial", "budget",
                 "free_list", "free_count", "n_live", "page_format"]
        if self.offload_pages > 0:
            names += list(self.OFFLOAD_BUFFERS)
        for name in names:
            setattr(v, name, getattr(self, name).data_ptr())
        return v

    @staticmethod
    def to_pool_layout(k: torch.Tensor) -> torch.Tensor:
        """Keys [m][P][L][Hkv][d] of m pages -> the pool's page layout
        [m][L][Hkv][P/16][d/8][16][8] (memdecay.h)."""
        m, P, L, Hkv, d = k.shape
        return k.view(m, P // 16, 16, L, Hkv, d // 8, 8).permute(0, 3, 4, 1, 5, 2, 6).contiguous()

    @staticmethod
    def from_pool_layout(pages: torch.Tensor) -> torch.Tensor:
        """The inverse: pool pages [m][L][Hkv][P/16][d/8][16][8] (or the pool
        itself) -> keys [m][P][L][Hkv][d]."""
        m, L, Hkv, nb, db = pages.shape[:5]
        return pages.permute(0, 3, 5, 1, 2, 4, 6).reshape(m, nb * 16, L, Hkv, db * 8)

    @staticmethod
    def to_value_layout(v: torch.Tensor) -> torch.Tensor:
        """Values [m][P][L][Hkv][d] of m pages -> the value pool's page layout
        [m][L][Hkv][P/16][d/32][4][16][2][4] (memdecay.h)."""
        m, P, L, Hkv, d = v.shape
        return v.view(m, P // 16, 4, 4, L, Hkv, d // 32, 2, 16).permute(0, 4, 5, 1, 6, 2, 8, 7, 3).contiguous()

    @staticmethod
    def from_value_layout(pages: torch.Tensor) -> torch.Tensor:
        """The inverse: value pool pages -> values [m][P][L][Hkv][d]."""
        m, L, Hkv, nb, db = pages.shape[:5]
        return pages.permute(0, 3, 5, 8, 1, 2, 4, 7, 6).reshape(m, nb * 16, L, Hkv, db * 32)

    @staticmethod
    def to_code_layout(v: torch.Tensor):
        """Values [m][P][L][Hkv][d] of m pages -> their codes
        [m][L][Hkv][P/16][d/64][4][16][4][4] (uint8) and scales
        [m][L][Hkv][P/16] (memdecay.h)."""
        m, P, L, Hkv, d = v.shape
        x = v.float().view(m, P // 16, 16, L, Hkv, d)
        top = x.abs().amax((2, 5))
        # (by a tensor: a number's division may become a product with its reciprocal)
        scale = torch.where(torch.isfinite(top), top / torch.full_like(top, 448.0), math.nan)
        q = x / torch.where(scale > 0, scale, 1.0)[:, :, None, :, :, None]
        q = torch.where((scale > 0)[:, :, None, :, :, None], q, 0.0)
        codes = q.to(torch.float8_e4m3fn).view(torch.uint8).view(m, P // 16, 4, 4, L, Hkv, d // 64, 4, 16)
        return codes.permute(0, 4, 5, 1, 6, 2, 8, 7, 3).contiguous(), scale.permute(0, 2, 3, 1).contiguous()

    @staticmethod
    def from_code_layout(codes: torch.Tensor, scale: torch.Tensor) -> torch.Tensor:
        """The inverse but for the rounding: pages of codes and their scales ->
        float32 values [m][P][L][Hkv][d]."""
        m, L, Hkv, nb, half = codes.shape[:5]
        x = codes.contiguous().view(torch.float8_e4m3fn).float() * scale[..., None, None, None, None, None]
        return x.permute(0, 3, 5, 8, 1, 2, 4, 7, 6).reshape(m, nb * 16, L, Hkv, half * 64)

    @staticmethod
    def positions(region, P: int, region_aligned: bool) -> np.ndarray:
        """Slot position (page * P + offset) of each prompt token in the
        session's page sequence: consecutive, or with region-aligned pages a
        fresh page at every region change (the positions skipped are holes)."""
        reg = np.asarray(region, dtype=np.int64)
        n = reg.size
        if not region_aligned or n == 0:
            return np.arange(n, dtype=np.int64)
        pos = np.empty(n, dtype=np.int64)
        p = 0
        for i in range(n):
            if i > 0 and reg[i] != reg[i - 1] and p % P:
                p += P - p % P          # close the page at the region boundary
            pos[i] = p
            p += 1
        return pos

    @classmethod
    def pages_for(cls, region, P: int, region_aligned: bool) -> int:
        """Pages a prompt with these region codes takes."""
        n = len(region)
        return 0 if n == 0 else (int(cls.positions(region, P, region_aligned)[-1]) + P) // P

    def load_session(self, s: int, keys: torch.Tensor, region, page_ids: Sequence[int],
                     budget: int, clock: int, t_ins=None, region_aligned: bool = False):
        """Place a session's prompt: keys bf16 [n][L][Hkv][d] (device), region
        codes [n], physical page ids in logical order (as many as the layout
        takes: ceil(n / P), or with region-aligned pages one more per region
        change inside a page; ``pages_for``).  Token i gets t_ins = t_ref =
        t_ins[i] (default i) and importance 0; holes get the hole code."""
        P = self.P
        n = int(keys.shape[0])
        if len(region) != n:
            raise ValueError("need one region code per token")
        # (the keys first, so that a call that is refused leaves the session as it was)
        pos = self.positions(region, P, region_aligned)
        m = (int(pos[-1]) + P) // P if n else 0
        full = torch.zeros((m * P,) + tuple(keys.shape[1:]), dtype=torch.bfloat16, device=self.device)
        full[torch.as_tensor(pos, device=self.device)] = keys.to(self.device, torch.bfloat16)
        # [m][P][L][Hkv][d] -> [m][L][Hkv][P][d]
        pages = self.to_pool_layout(full.view(m, P, self.L, self.Hkv, self.d))
        ids, _, _ = self.place_session(s, region, page_ids, budget, clock, t_ins, region_aligned)
        self.k_pool.index_copy_(0, ids, pages)

    def place_session(self, s: int, region, page_ids: Sequence[int], budget: int, clock: int, t_ins=None,
                      region_aligned: bool = False):
        """load_session without its keys, for a prompt whose rows come through
        MemDecay.write_rows: the page table, the counts and every token's
        region and times.  Returns the page ids, the slot of each token
        (``positions``) and the number of pages."""
        P = self.P
        n = len(region)
        pos = self.positions(region, P, region_aligned)
        n_pos = int(pos[-1]) + 1 if n else 0
        m = (n_pos + P - 1) // P
        if len(page_ids) != m or m > self.max_pages:
            raise ValueError("need one page id per page of the layout, within max_pages")
        if t_ins is not None and len(t_ins) != n:
            raise ValueError("need one time per token")
        ids = torch.as_tensor(np.asarray(page_ids, dtype=np.int64), device=self.device)
        posd = torch.as_tensor(pos, device=self.device)
        reg = torch.as_tensor(np.asarray(region, dtype=np.uint8), device=self.device)
        t0 = torch.arange(n, dtype=torch.int32, device=self.device) if t_ins is None else \
            torch.as_tensor(np.asarray(t_ins, dtype=np.int32), device=self.device)
        slots = (ids.view(-1, 1) * P + torch.arange(P, device=self.device).view(1, -1)).view(-1)
        used = slots[:n_pos]
        self.region.view(-1)[used] = B.MD_REGION_HOLE
        self.t_ins.view(-1)[used] = 0
        self.t_ref.view(-1)[used] = 0
        self.importance.view(-1)[used] = 0.0
        flat = slots[posd]
        self.region.view(-1)[flat] = reg
        self.t_ins.view(-1)[flat] = t0
        self.t_ref.view(-1)[flat] = t0
        self.importance.view(-1)[flat] = 0.0
        self.page_format[ids] = 0
        self.page_table[s, :m] = ids.to(torch.int32)
        self.page_table[s, m:] = -1
        self.page_serial[s, :m] = torch.arange(m, dtype=torch.int32, device=self.device)
        self.page_serial[s, m:] = -1
        self.n_pages[s] = m
        self.n_tokens[s] = n_pos
        self.n_live[s] = n
        self.clock[s] = clock
        self.next_serial[s] = m
        self.budget[s] = budget
        if self.v_held is not None:
            self.v_held[s] = -1
        return ids, posd, m

    def place_tokens(self, s: int, region, region_aligned: bool = False) -> np.ndarray:
        """Room for more tokens of a session in use, as steps would append them
        one by one (a chunk of a prompt, tokens to verify): their region codes
        [n], their times from the session's clock on, and the pages that they
        open, off the free list.  Their keys and values come through
        MemDecay.write_rows.  Returns their slots."""
        P, region = self.P, np.asarray(region, dtype=np.uint8)
        n, nt, np_, clock = len(region), int(self.n_tokens[s]), int(self.n_pages[s]), int(self.clock[s])
        if self.offload_pages > 0:
            raise ValueError("tokens are not placed beside an offload tier")
        if n == 0:
            return np.zeros(0, np.int64)
        old = self.page_table[s, :np_].cpu().numpy()
        pos = np.arange(nt, nt + n)
        if region_aligned:
            ahead = nt % P   # the open page's tokens, the last one's region among them
            last = [int(self.region[int(old[-1]), ahead - 1])] * ahead if ahead else []
            pos = nt - ahead + self.positions(np.concatenate([np.array(last, np.uint8), region]), P, True)[ahead:]
        end, free = int(pos[-1]) + 1, int(self.free_count[0])
        m = -(-end // P)
        if m > self.max_pages or m - np_ > free:
            raise ValueError(f"{m - np_} more pages for session {s} with {np_} of {self.max_pages}, {free} pages are free")
        ids = self.free_list[free - (m - np_):free].flip(0)
        self.free_count[0] = free - (m - np_)
        self.page_table[s, np_:m] = ids
        serial = int(self.next_serial[s])
        self.page_serial[s, np_:m] = torch.arange(serial, serial + m - np_, dtype=torch.int32, device=self.device)
        self.next_serial[s] = serial + m - np_
        self.page_format[ids.long()] = 0
        table = self.page_table[s, :m].long()
        flat = lambda at: table[torch.as_tensor(at // P, device=self.device)] * P + torch.as_tensor(at % P, device=self.device)
        every, own = flat(np.arange(nt, end)), flat(pos)
        t = torch.arange(clock + 1, clock + 1 + n, dtype=torch.int32, device=self.device)
        for x, hole, token in ((self.region, B.MD_REGION_HOLE, torch.as_tensor(region, device=self.device)), (self.t_ins, 0, t),
                               (self.t_ref, 0, t), (self.importance, 0.0, 0.0)):
            x.view(-1)[every] = hole
            x.view(-1)[own] = token
        self.n_pages[s] = m
        self.n_tokens[s] = end
        self.n_live[s] += n
        self.clock[s] = clock + n
        return pos

    def take_back(self, s: int, n: int):
        """The last n tokens of a session leave (of tokens to verify, those that
        failed): the pages that they alone were in go back to the free list,
        and the clock to where it was before them."""
        P, nt, np_ = self.P, int(self.n_tokens[s]), int(self.n_pages[s])
        table = self.page_table[s, :np_].long()
        live = np.flatnonzero((self.region[table].flatten()[:nt] != B.MD_REGION_HOLE).cpu().numpy())
        if self.offload_pages > 0 or n < 0 or n > len(live):
            raise ValueError(f"{n} of {len(live)} tokens of session {s} to take back")
        if n == 0:
            return
        left = int(live[-n - 1]) + 1 if n < len(live) else 0
        m = -(-left // P)
        if left < m * P and int(self.page_format[table[m - 1]]):
            raise ValueError(f"the page that session {s} would go on in holds 8-bit keys")
        free = int(self.free_count[0])
        self.free_list[free:free + np_ - m] = self.page_table[s, m:np_].flip(0)
        self.free_count[0] = free + np_ - m
        self.page_table[s, m:] = -1
        self.page_serial[s, m:] = -1
        self.n_pages[s] = m
        self.n_tokens[s] = left
        self.n_live[s] -= n
        self.clock[s] -= n

    def load_values(self, s: int, values: torch.Tensor, region=None):
        """Place the values bf16 [n][L][Hkv][d] of a session's prompt next to
        the keys that ``load_session`` placed, one for each of its tokens;
        region: the same codes, with region-aligned pages only."""
        n, P = int(values.shape[0]), self.P
        if self.v_pool is None and self.v_codes is None:
            raise ValueError("the cache has no values (PagedCache(values=True))")
        if region is not None and len(region) != n:
            raise ValueError("need one region code per token")
        pos = self.positions(np.zeros(n) if region is None else region, P, region is not None)
        slots = int(pos[-1]) + 1 if n else 0
        if slots != int(self.n_tokens[s]) or (region is not None and n != int(self.n_live[s])):
            raise ValueError(f"{n} values in {slots} slots for session {s} with {int(self.n_tokens[s])} slots in use")
        if n == 0:
            return
        m = (slots + P - 1) // P
        full = torch.zeros((m * P,) + tuple(values.shape[1:]), dtype=torch.bfloat16, device=self.device)
        full[torch.as_tensor(pos, device=self.device)] = values.to(self.device, torch.bfloat16)
        ids = self.page_table[s, :m].long()
        full = full.view(m, P, self.L, self.Hkv, self.d)
        if self.v_pool is not None:
            self.v_pool.index_copy_(0, ids, self.to_value_layout(full))
            return
        codes, scale = self.to_code_layout(full)
        self.v_codes.index_copy_(0, ids, codes)
        self.v_scale.index_copy_(0, ids, scale)
        at = (slots - 1) % P // 16 * 16
        self.v_open[s] = full[-1, at:at + 16].permute(1, 2, 0, 3)
        if self.v_held is not None:
            self.v_held[s] = -1
            self.v_held[s, ..., 0] = (ids[-1] * (P // 16) + at // 16).int()
            self.v_held[s, ..., 1] = (slots - 1) % 16 + 1

    def set_free_pages(self, ids: Sequence[int]):
        """The free list: ids pop from the end."""
        ids = np.ascontiguousarray(ids, dtype=np.int32)
        self.free_list.zero_()
        if ids.size:
            self.free_list[: ids.size] = torch.as_tensor(ids, device=self.device)
        self.free_count[0] = int(ids.size)


class MemDecay:
    """A library handle bound to a PagedCache, with the step's output buffers."""

    def __init__(self, cache: PagedCache, base_priority: torch.Tensor, decay_rate: torch.Tensor, *,
                 rho: float, alpha: float, tau_scale: float, pinned_mask: int,
                 n_regions: int = 7, stream: Optional[torch.cuda.Stream] = None,
                 fused: Optional[bool] = None, attention_norm: bool = False, window: int = 1,
                 region_aligned: bool = False, quant_threshold: float = 0.0, static: bool = False,
                 drop_threshold: float = 0.0, cooperative: bool = False, row_groups: bool = True):
        # fused: True = always the fused kernel, False = always the
        # multi-kernel path, None = the library picks from the cache's sizes;
        # cooperative: the fused kernel as a cooperative launch (for a GPU
        # shared with other streams); row_groups: False keeps every fused
        # unit on all rows
        self.cache = cache
        dev = cache.device
        self.b = base_priority.to(dev, torch.float32).contiguous()
        self.lam = decay_rate.to(dev, torch.float32).contiguous()
        cfg = B.md_config(n_layers=cache.L, n_q_heads=cache.Hq, n_kv_heads=cache.Hkv,
                          head_dim=cache.d, page_size=cache.P, max_sessions=cache.S,
                          max_pages=cache.max_pages, n_phys_pages=cache.n_phys,
                          n_regions=n_regions, pinned_region_mask=pinned_mask, rho=rho,
                          alpha=alpha, tau_scale=tau_scale,
                          flags=(0 if fused is None else (B.MD_FLAG_FUSED if fused else B.MD_FLAG_NO_FUSED))
                          | (B.MD_FLAG_NORM_ATTENTION if attention_norm else 0)
                          | (B.MD_FLAG_REGION_ALIGNED if region_aligned else 0)
                          | (B.MD_FLAG_COOPERATIVE if cooperative else 0)
                          | (0 if row_groups else B.MD_FLAG_NO_ROW_GROUPS),
                          window=window, quant_threshold=quant_threshold,
                          offload_pages=cache.offload_pages, drop_threshold=drop_threshold)
        rp = B.md_region_params(base_priority=self.b.data_ptr(), decay_rate=self.lam.data_ptr())
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)
        self._cfg, self._rp, self._cv = cfg, rp, cache.view()
        # static: md_init_static (the library's static scratch, no allocation)
        init = B.md_init_static if static else B.md_init
        self.handle = init(cfg, rp, self._cv, self.stream.cuda_stream)
        S, MP = cache.S, cache.max_pages
        self.page_score = torch.zeros((S, MP), dtype=torch.float32, device=dev)
        self.evict_serial = torch.zeros((S, MP), dtype=torch.int32, device=dev)
        self.evict_count = torch.zeros(S, dtype=torch.int32, device=dev)
        self.infeasible = torch.zeros(S, dtype=torch.uint8, device=dev)

        # work space of the decode operators (one per handle: calls on its
        # stream run one after another)
        self._attend_ws = self._select_ws = self._rows_ws = None
        self._device = cache.k_pool.get_device()
        self._held = None   # the handle's md_open_blocks
        if cache.v_pool is not None or cache.v_codes is not None:   # now, so that a captured call allocates nothing
            self._workspace(True)
        if cache.key_bounds is not None:
            self._workspace(False)

    def _workspace(self, attend: bool) -> torch.Tensor:
        ws = self._attend_ws if attend else self._select_ws
        if ws is None:
            n = B.md_decode_workspace(self.handle)[0 if attend else 1]
            with torch.cuda.stream(self.stream):
                ws = torch.zeros(max(n, 16), dtype=torch.uint8, device=self.cache.device)
            if attend:
                self._attend_ws = ws
            else:
                self._select_ws = ws
        return ws

    # ---- the four calls of one step
    def observe(self, step: int, q: torch.Tensor, new_k: Optional[torch.Tensor] = None,
                new_region: Optional[torch.Tensor] = None, abar_out: Optional[torch.Tensor] = None):
        B.md_observe_step(self.handle, step, None if q is None else _ptr(q, torch.float32),
                          None if new_k is None else _ptr(new_k, torch.bfloat16),
                          None if new_region is None else _ptr(new_region, torch.uint8),
                          None if abar_out is None else _ptr(abar_out, torch.float32))

    def score(self, token_score: Optional[torch.Tensor] = None, page_score: bool = True):
        B.md_score_pages(self.handle, self.page_score.data_ptr() if page_score else None,
                         None if token_score is None else _ptr(token_score, torch.float32))

    def select(self):
        B.md_select_evict(self.handle, self.evict_serial.data_ptr(), self.evict_count.data_ptr(),
                          self.infeasible.data_ptr())

    def compact(self, evict_serial: Optional[torch.Tensor] = None,
                evict_count: Optional[torch.Tensor] = None):
        """Apply this step's selection (no arguments), or the given lists."""
        if evict_serial is None and evict_count is None:
            B.md_compact(self.handle, None, None)
        else:
            B.md_compact(self.handle, _ptr(evict_serial, torch.int32), _ptr(evict_count, torch.int32))

    def select_compact(self):
        """select() then compact() with this step's selection, as one call
        (one launch when no tier is configured)."""
        B.md_select_compact(self.handle, self.evict_serial.data_ptr(), self.evict_count.data_ptr(),
                            self.infeasible.data_ptr())

    def step(self, step: int, q, new_k=None, new_region=None, page_scores: bool = True):
        """One decode step; page_scores=False leaves self.page_score untouched
        (the library still scores every page for its own selection).  The
        step's selection is applied as it stands (select_compact)."""
        self.observe(step, q, new_k, new_region)
        if q is None:   # a decode step without an observation only appends
            return
        self.score(page_score=page_scores)
        self.select_compact()

    # ---- what a decode engine runs around the step (memdecay.h).  A call of
    # a few sessions takes the device less than 10 us, so the checks keep to
    # comparisons of the tensors' shapes, strides, types and devices.
    # Like the step's calls they run on the stream that the handle was made
    # with (``MemDecay(stream=...)``), whatever stream is current: tensors made
    # or read on another one need a wait in between.
    def norm_rope(self, qkv: torch.Tensor, q_out: torch.Tensor, k_out: torch.Tensor,
                  v_out: Optional[torch.Tensor] = None, *, q_weight: Optional[torch.Tensor] = None,
                  k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  inv_freq: Optional[torch.Tensor] = None, position: Optional[torch.Tensor] = None,
                  interleaved: bool = False):
        """Norms of the query and key heads and their rotation by position.

        qkv [n][(Hq + 2 Hkv) d] float32, bfloat16 or float16 rows; q_out
        float32 [n][Hq][d]; k_out, v_out bfloat16 [n][Hkv][d].  Rows may be
        any distance apart (a layer of the step's q and new_k buffers).
        q_weight, k_weight [d]: None leaves those heads as they are.
        inv_freq float64 [r / 2]: the first r elements of each head turn (None:
        none).  position int32 [n]; None: each session's clock (n = S).  Runs
        on the handle's stream, whatever stream is current."""
        c, dev = self.cache, self._device
        n = qkv.shape[0]
        if qkv.dtype not in TYPES:
            raise ValueError(f"expected float32, bfloat16 or float16 rows, got {qkv.dtype}")
        if n == 0:
            return
        qkv_at, qkv_pitch = _rows(qkv, qkv.dtype, n, c.Hq + 2 * c.Hkv, c.d, dev)
        q_at, q_pitch = _rows(q_out, torch.float32, n, c.Hq, c.d, dev)
        k_at, kv_pitch = _rows(k_out, torch.bfloat16, n, c.Hkv, c.d, dev)
        v_at = 0
        if v_out is not None:
            v_at, v_pitch = _rows(v_out, torch.bfloat16, n, c.Hkv, c.d, dev)
            if v_pitch != kv_pitch:
                raise ValueError("k_out and v_out have rows the same distance apart")
        B.md_norm_rope(self.handle, B.ROPE_ARGS.pack(
            qkv_at, qkv_pitch, TYPES[qkv.dtype], n,
            0 if q_weight is None else _flat(q_weight, torch.float32, c.d, dev),
            0 if k_weight is None else _flat(k_weight, torch.float32, c.d, dev), eps,
            0 if inv_freq is None else 2 * inv_freq.numel(),
            0 if inv_freq is None else _flat(inv_freq, torch.float64, inv_freq.numel(), dev),
            0 if position is None else _flat(position, torch.int32, n, dev), int(interleaved), q_at, q_pitch, k_at, v_at,
            kv_pitch))

    def append_values(self, new_v: torch.Tensor):
        """The values bf16 [S][L][Hkv][d] of the tokens that the last observe
        appended (before anything is compacted); in a cache of 8-bit values
        they become codes.  Runs on the handle's stream, whatever stream is
        current."""
        c = self.cache
        new_at = _flat(new_v, torch.bfloat16, c.S * c.L * c.Hkv * c.d, self._device)
        if c.v_codes is not None:
            B.md_append_codes(self.handle, new_at, B.VALUES.pack(*self._value_pools(True)))
        else:
            B.md_append_values(self.handle, new_at, self._values())

    def _values(self) -> int:
        v = self.cache.v_pool
        if v is None:
            raise ValueError("the cache has no values (PagedCache(values=True))")
        return _flat(v, torch.bfloat16, self.cache.k_pool.numel(), self._device)

    def _value_pools(self, written: bool):
        """The fields of md_values."""
        c, dev = self.cache, self._device
        if c.v_codes is None:
            return self._values(), 0, 0, 0
        n = c.k_pool.numel()
        if written and self._held is not c.v_held:
            self._keep_open_blocks()
        return (0, _flat(c.v_codes, torch.uint8, n, dev), _flat(c.v_scale, torch.float32, n // (16 * c.d), dev),
                _flat(c.v_open, torch.bfloat16, c.S * c.L * c.Hkv * 16 * c.d, dev) if written else 0)

    def _keep_open_blocks(self):
        """Tells the handle where the cache keeps what its open blocks hold."""
        c, dev = self.cache, self._device
        if c.v_held is None:
            B.md_open_blocks(self.handle, None, None)
        else:
            n = c.S * c.L * c.Hkv
            B.md_open_blocks(self.handle, _flat(c.v_before, torch.bfloat16, 16 * n * c.d, dev),
                             _flat(c.v_held, torch.int32, 4 * n, dev))
        self._held = c.v_held

    # ---- rows of the cache: prompts, chunks of them, tokens to verify.  The
    # rows of a call are ragged: row_start int32 [S + 1] tells where each
    # session's begin, row_slot int32 [n] their slots (None: each session's
    # last ones), which PagedCache.place_session has set up.  The tensors stay
    # on the device; a row that is not in its session's slots counts as not
    # there (device_status() tells of it).
    def _row_list(self, n: int, row_start: torch.Tensor, row_slot: Optional[torch.Tensor]):
        dev = self._device
        return (_flat(row_start, torch.int32, self.cache.S + 1, dev),
                0 if row_slot is None else _flat(row_slot, torch.int32, n, dev), n, 0)

    def _kv_rows(self, k, v, dtypes):
        """Rows, addresses, distance and type of keys and values [n][Hkv][d], either of which may be left out."""
        c, dev = self.cache, self._device
        one = k if k is not None else v
        if one is None:
            raise ValueError("rows of keys, of values, or both")
        n, dtype = one.shape[0], one.dtype
        if dtype not in dtypes:
            raise ValueError(f"expected {' or '.join(map(str, dtypes))} rows, got {dtype}")
        k_at = v_at = 0
        pitches = []
        for x in (k, v):
            if x is not None:
                at, pitch = _rows(x, dtype, n, c.Hkv, c.d, dev)
                pitches.append(pitch)
                if x is k:
                    k_at = at
                if x is v:
                    v_at = at
        if len(set(pitches)) > 1:
            raise ValueError("keys and values have rows the same distance apart")
        return n, k_at, v_at, pitches[0], dtype

    def write_rows(self, layer: int, row_start: torch.Tensor, k: Optional[torch.Tensor] = None,
                   v: Optional[torch.Tensor] = None, *, row_slot: Optional[torch.Tensor] = None):
        """Keys and values bf16 [n][Hkv][d] (rows any distance apart) of one
        layer into the pools, values as codes in a cache of 8-bit values.  A
        session's slots ascend, and its rows are written in order; rows whose
        slot is not there (-1) may lie among them.  Keys of pages that hold
        8-bit keys are left alone.  Page bounds do not follow: behind it
        update_bounds(True).  k and v have rows the same distance apart.  Runs
        on the handle's stream, whatever stream is current.

        Of tokens to verify (PagedCache.place_tokens) the last ones may leave
        again (PagedCache.take_back): with 8-bit values rows and steps then go on
        inside the last block of 16 slots or the one before it; further back,
        from a block's first slot (else they do not count: device_status())."""
        n, k_at, v_at, pitch, _ = self._kv_rows(k, v, (torch.bfloat16,))
        rows = self._row_list(n, row_start, row_slot)
        if n == 0:
            return
        B.md_write_rows(self.handle, layer, B.WRITE_ARGS.pack(
            *rows, k_at, v_at, pitch, *((0, 0, 0, 0) if v is None else self._value_pools(True))))

    def read_rows(self, layer: int, row_start: torch.Tensor, k_out: Optional[torch.Tensor] = None,
                  v_out: Optional[torch.Tensor] = None, *, row_slot: Optional[torch.Tensor] = None):
        """Keys and values of one layer out of the pools into k_out and v_out
        [n][Hkv][d], bfloat16 or float32, rows any distance apart: what 8-bit
        codes stand for, bf16 ones as they are.  Runs on the handle's stream,
        whatever stream is current."""
        n, k_at, v_at, pitch, dtype = self._kv_rows(k_out, v_out, (torch.bfloat16, torch.float32))
        rows = self._row_list(n, row_start, row_slot)
        if n == 0:
            return
        B.md_read_rows(self.handle, layer, B.READ_ARGS.pack(
            *rows, k_at, v_at, pitch, TYPES[dtype], *((0, 0, 0, 0) if v_out is None else self._value_pools(False))))

    def attend_rows(self, layer: int, q: torch.Tensor, out: torch.Tensor, row_start: torch.Tensor, *,
                    row_slot: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                    lse: Optional[torch.Tensor] = None):
        """Attention of rows [n][Hq][d] over their sessions' cached tokens up to
        their own (write_rows comes first); with window > 0 over those less
        than ``window`` slots back and the first ``sinks`` slots (of the cache
        as it stands, as in attend).  q and out float32
        or bfloat16, rows any distance apart, lse float32 [n][Hq].  bf16 q and
        out take the faster products; float32 on either side the exact ones.
        Runs on the handle's stream, whatever stream is current, in a work
        space of the handle's, so that captured calls of it are not replayed
        at the same time; the first call allocates it and is not captured."""
        c, dev = self.cache, self._device
        n = q.shape[0]
        if q.dtype not in (torch.float32, torch.bfloat16) or out.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"expected float32 or bfloat16 queries and outputs, got {q.dtype} and {out.dtype}")
        q_at, q_pitch = _rows(q, q.dtype, n, c.Hq, c.d, dev)
        out_at, out_pitch = _rows(out, out.dtype, n, c.Hq, c.d, dev)
        rows = self._row_list(n, row_start, row_slot)
        lse_at = 0 if lse is None else _flat(lse, torch.float32, n * c.Hq, dev)
        pools = self._value_pools(False)
        if n == 0:
            return
        if self._rows_ws is None:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("attend_rows allocates its work space in its first call: make one before the capture")
            with torch.cuda.stream(self.stream):
                self._rows_ws = torch.zeros(max(B.md_rows_workspace(self.handle), 16), dtype=torch.uint8, device=c.device)
        B.md_attend_rows(self.handle, layer, B.ROWS_ARGS.pack(
            *rows, q_at, q_pitch, TYPES[q.dtype], TYPES[out.dtype], out_at, out_pitch, lse_at, window, sinks, *pools,
            self._rows_ws.data_ptr()))

    def attend(self, layer: int, q: torch.Tensor, out: torch.Tensor, *, new_k: Optional[torch.Tensor] = None,
               new_v: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               blocks: Optional[torch.Tensor] = None, block_count: Optional[torch.Tensor] = None, window: int = 0,
               sinks: int = 0):
        """Attention of one token of every session in one layer over its
        cached tokens (or the listed pages) and, with new_k and new_v bf16
        [S][Hkv][d], itself.  q float32 and out (float32 or bfloat16)
        [S][Hq][d], lse float32 [S][Hq]; sessions of q, out and of the new
        keys and values may be any distance apart.  A row's listed pages
        ascend (device_status() tells of one that does not).  Runs on the
        handle's stream, whatever stream is current; the handle has one work
        space, so captured calls of it are not replayed at the same time.
        With window > 0 the token (the slot behind the session's last, or
        without new_k the last one) sees the slots less than ``window`` back
        and the first ``sinks`` ones; not together with blocks.  Slots are those
        of the cache as it stands, holes among them: behind an eviction a window
        reaches further back in the text, and other slots are the first."""
        c, dev = self.cache, self._device
        S = c.S
        q_at, q_pitch = _rows(q, torch.float32, S, c.Hq, c.d, dev)
        if out.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"expected float32 or bfloat16 outputs, got {out.dtype}")
        out_at, out_pitch = _rows(out, out.dtype, S, c.Hq, c.d, dev)
        k_at = v_at = kv_pitch = 0
        if new_k is not None:
            k_at, kv_pitch = _rows(new_k, torch.bfloat16, S, c.Hkv, c.d, dev)
        if new_v is not None:
            v_at, v_pitch = _rows(new_v, torch.bfloat16, S, c.Hkv, c.d, dev)
            if new_k is not None and v_pitch != kv_pitch:
                raise ValueError("new_k and new_v have sessions the same distance apart")
        if blocks is None and block_count is not None:
            raise ValueError("counts without their blocks")
        b_at, n_at, most = (0, 0, 0) if blocks is None else self._lists(blocks, block_count)
        pools = (self._values(),) if c.v_codes is None else self._value_pools(False)
        args = B.ATTEND_ARGS.pack(
            q_at, q_pitch, k_at, v_at, kv_pitch, pools[0], b_at, n_at, most, TYPES[out.dtype], out_at, out_pitch,
            0 if lse is None else _flat(lse, torch.float32, S * c.Hq, dev), self._workspace(True).data_ptr())
        if window == 0 and len(pools) == 1:
            B.md_attend_token(self.handle, layer, args)
        else:
            B.md_attend_values(self.handle, layer, args, B.VALUES.pack(*pools, *(0,) * (4 - len(pools))), window, sinks)

    def _lists(self, blocks: torch.Tensor, count: torch.Tensor):
        c, dev = self.cache, self._device
        # (an empty tensor's address is 0, which the library takes for no list: every page)
        if count is None or blocks.dim() != 3 or blocks.shape[0] != c.S or blocks.shape[1] != c.Hkv or blocks.shape[2] < 1:
            raise ValueError("blocks hold [S][Hkv][max_blocks], max_blocks >= 1, their counts [S][Hkv]")
        return _flat(blocks, torch.int32, blocks.numel(), dev), _flat(count, torch.int32, c.S * c.Hkv, dev), blocks.shape[2]

    def _bounds(self):
        c, dev = self.cache, self._device
        if c.key_bounds is None or c.bound_exp is None:
            raise ValueError("the cache has no bounds (PagedCache(bounds=True))")
        n = c.n_phys * c.L * c.Hkv
        return _flat(c.key_bounds, torch.int8, 2 * n * c.d, dev), _flat(c.bound_exp, torch.int8, n, dev)

    def update_bounds(self, all_pages: bool = False):
        """Bounds of the keys, once per step behind its compaction: of each
        session's last page and, with the quantised tier, of the pages that
        became codes since the last call; or of every page (after the prompts
        are loaded, and behind write_rows; also faster where most of a cache has become codes).
        Runs on the handle's stream, whatever stream is current."""
        B.md_key_bounds(self.handle, int(all_pages), *self._bounds())

    def select_blocks(self, layer: int, q: torch.Tensor, blocks: torch.Tensor, block_count: torch.Tensor, *,
                      first: int = 1, last: int = 1):
        """The pages each session's query q float32 [S][Hq][d] attends to in
        one layer: blocks int32 [S][Hkv][max_blocks], block_count int32
        [S][Hkv]; always the ``first`` and ``last`` pages of the session.  Runs
        on the handle's stream, whatever stream is current, in the handle's
        one work space."""
        c = self.cache
        q_at, q_pitch = _rows(q, torch.float32, c.S, c.Hq, c.d, self._device)
        b_at, n_at, most = self._lists(blocks, block_count)
        bounds, exp = self._bounds()
        B.md_select_blocks(self.handle, layer, B.SELECT_ARGS.pack(q_at, q_pitch, bounds, exp, first, last, most, b_at, n_at,
                                                                 self._workspace(False).data_ptr()))

    def calib_accumulate(self, abar: torch.Tensor, bucket_steps: int, stats) -> None:
        """Add this observation to stats = (mass_fx, count, age_sum), int64
        tensors [S][n_regions][n_buckets] viewed as uint64 by the library."""
        mass, count, age = stats
        B.md_calib_accumulate(self.handle, _ptr(abar, torch.float32), bucket_steps, mass.shape[-1],
                              mass.data_ptr(), count.data_ptr(), age.data_ptr())

    def device_status(self, with_warning: bool = False):
        return B.md_read_device_status(self.handle, with_warning)

    def profile(self, kernels=("logits",)):
        """Time the named kernels with events from now on (() turns it off)."""
        mask = 0
        for k in kernels:
            mask |= 1 << B.KERNELS.index(k)
        B.md_profile_enable(self.handle, mask)

    def profile_read(self, kernel: str):
        return B.md_profile_read(self.handle, B.KERNELS.index(kernel))

    def counters(self):
        return B.md_read_counters(self.handle)

    def kernel_config(self) -> dict:
        return B.md_kernel_config(self.handle)

    def observe_path(self) -> dict:
        return B.md_observe_path(self.handle)

    def close(self):
        if self.handle is not None:
            B.md_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _ptr(t: torch.Tensor, dtype) -> int:
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"expected a contiguous {dtype} tensor, got {t.dtype}")
    return t.data_ptr()



TYPES = {torch.float32: B.MD_F32, torch.bfloat16: B.MD_BF16, torch.float16: B.MD_F16}


def _rows(t: torch.Tensor, dtype, n: int, heads: int, d: int, device: int):
    """Address of t, n rows [heads][d] (or [heads d]) each contiguous, and the
    elements between them."""
    shape, stride = t.shape, t.stride()
    if shape == (n, heads, d):
        rows = stride[2] == 1 and (stride[1] == d or heads == 1)
    else:
        rows = shape == (n, heads * d) and stride[1] == 1
    if not rows or t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"expected {dtype} [{n}][{heads}][{d}] with contiguous rows on device {device}, got {t.dtype} "
                         f"{tuple(shape)} with strides {stride} on {t.device}")
    return t.data_ptr(), stride[0] if n > 1 else heads * d


def _flat(t: torch.Tensor, dtype, n: int, device: int) -> int:
    """Address of t, n contiguous elements."""
    if t.dtype is not dtype or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"expected {n} contiguous elements of {dtype} on device {device}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()
