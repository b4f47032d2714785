"""Page bounds and the quantised tier: a key that becomes an 8-bit code moves
by up to 2^-4 of itself, so the bounds of a page that the compaction converts
are those of its codes after the next update, and a page's score is again no
less than its logits (but for the query's rounding).

Bounds are whole numbers: equal to the oracle's of the keys that the pages
hold, codes as the float32 product of scale and code.
"""
import numpy as np
import pytest
import torch

import decode_oracle as O
from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import MemDecay, PagedCache
from test_gpu_decode import BF16, D, World, say

pytestmark = pytest.mark.gpu


def page_keys(c, p):
    """Keys float32 [P][L][Hkv][d] of a physical page as they are stored."""
    if not int(c.page_format[p]):
        return PagedCache.from_pool_layout(c.k_pool[p:p + 1])[0].float().cpu()
    raw = c.k_pool[p].contiguous().view(torch.uint8).view(c.L, c.Hkv, c.P // 16, 4096).cpu()
    t, e = torch.arange(16)[:, None], torch.arange(D)[None]
    code = raw[..., 1024 * (e // 64) + 16 * (t + 16 * ((e // 8) % 4)) + 8 * ((e // 32) % 2) + e % 8]
    scale = raw[..., 2048:2052].contiguous().view(torch.float32)
    keys = code.view(torch.float8_e4m3fn).float() * scale[..., None]        # [L][Hkv][block][16][d]
    return keys.flatten(2, 3).permute(2, 0, 1, 3)


def wrong_bounds(c, only_codes=False):
    """(session, page) whose bounds are not those of the keys it holds."""
    table, npg, ntok = c.page_table.cpu().numpy(), c.n_pages.cpu().numpy(), c.n_tokens.cpu().numpy()
    region, fmt = c.region.cpu().numpy(), c.page_format.cpu().numpy()
    got, exp = c.key_bounds.cpu().numpy(), c.bound_exp.cpu().numpy()
    bad = []
    for s in range(c.S):
        for o in range(npg[s]):
            p = int(table[s, o])
            if only_codes and not fmt[p]:
                continue
            live = [j for j in range(c.P) if o * c.P + j < ntok[s] and region[p, j] != B.MD_REGION_HOLE]
            k = page_keys(c, p)[live].numpy()
            ok = True
            for layer in range(c.L):
                for kv in range(c.Hkv):
                    lo, hi, e = O.bounds(k[:, layer, kv])
                    ok &= exp[p, layer, kv] == e and (got[p, layer, kv, 0] == lo).all() and (got[p, layer, kv, 1] == hi).all()
            if not ok:
                bad.append((s, o))
    return bad


def make(P=16, aligned=False, static=False, stream=None, seed=31, shape=(3, 4, 2)):
    by = P // 16   # sessions and budgets of as many pages
    w = World(*shape, P, [150 * by, 0, 97 * by, 333 * by], seed=seed, aligned=aligned, extra=40, spare=40, quant=1e-9,
              static=static, stream=stream)
    w.cache.budget.copy_(torch.tensor([90, 60, 97, 200], dtype=torch.int32) * by)
    w.md.update_bounds(all_pages=True)
    return w


def step(w, i, before=False):
    """One step up to its compaction; before: the bounds are updated before
    it, so that those of the pages that it converts are due at the next."""
    c, md = w.cache, w.md
    q, nk = w.normal(c.S, 1, c.L, c.Hq, D), w.normal(c.S, c.L, c.Hkv, D, dtype=BF16)
    region = torch.full((c.S,), i // 6 % 7, dtype=torch.uint8, device=w.dev)
    torch.cuda.synchronize()
    md.observe(i, q, nk, region)
    md.score()
    if before:
        md.update_bounds()
    md.select_compact()
    torch.cuda.synchronize()   # (the step's inputs live until here, whatever stream the handle has)


@pytest.mark.parametrize("kw", [dict(), dict(P=64), dict(aligned=True), dict(static=True)], ids=str)
def test_bounds_follow_pages_into_codes(kw):
    say("[codes]", kw)
    w = make(**kw)
    c, md = w.cache, w.md
    moved = 0
    for i in range(1, 31):
        step(w, i, before=i % 5 == 0)
        moved += len(wrong_bounds(c, only_codes=True))
        if i % 5:
            md.update_bounds()
            torch.cuda.synchronize()
            assert wrong_bounds(c) == [], i
    assert int(c.page_format.sum()) > 0 and moved > 0    # pages were converted, and their bounds had to move
    assert md.device_status() == 0


def test_bounds_of_codes_without_room_for_their_times():
    # a static handle whose pages' times of conversion would not fit the static scratch
    # (only the handle is told of that many pages; none of them is used)
    w = make(seed=32, shape=(1, 1, 1))
    c, ones = w.cache, torch.ones((4, 7))
    w.md.close()
    pages, c.n_phys = c.n_phys, 40 << 20
    w.md = MemDecay(c, ones, ones * 0.01, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0, quant_threshold=0.3, static=True,
                    fused=True)
    c.n_phys = pages
    w.md.update_bounds(all_pages=True)
    for i in range(1, 13):
        step(w, i)
        w.md.update_bounds()
        torch.cuda.synchronize()
        assert wrong_bounds(c) == [], i
    assert int(c.page_format.sum()) > 0 and w.md.device_status() == 0
    w.md.close()


def test_captured_update_follows_pages_into_codes():
    side = torch.cuda.Stream()
    w = make(stream=side, seed=33)
    torch.cuda.synchronize()
    w.md.update_bounds()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        w.md.update_bounds()
    for i in range(1, 13):
        step(w, i)
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert wrong_bounds(w.cache) == [], i
    assert int(w.cache.page_format.sum()) > 0 and w.md.device_status() == 0


def test_scores_hold_for_pages_of_codes():
    # whole queries that need no rounding: no key of a page beats its score
    w = make(seed=34)
    c = w.cache
    for i in range(1, 8):
        step(w, i)
        w.md.update_bounds()
    torch.cuda.synchronize()
    rng = np.random.default_rng(3)
    q = rng.integers(-127, 128, (2, D)).astype(np.float64)
    q[:, 0] = 127
    seen = 0
    for s in range(c.S):
        for o in range(int(c.n_pages[s])):
            p = int(c.page_table[s, o])
            if int(c.page_format[p]):
                k = page_keys(c, p)[:, 1, 0].numpy().astype(np.float64)
                lo, hi = c.key_bounds[p, 1, 0].cpu().numpy().astype(np.int64)
                assert O.block_score(q, lo, hi, int(c.bound_exp[p, 1, 0])) >= (k @ q.T).max()
                seen += 1
    assert seen > 0
