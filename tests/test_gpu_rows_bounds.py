"""Page bounds and windows around rows that enter the cache: the bounds of
every page are due behind them, and windows count the slots that there are."""
import math

import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import MemDecay, PagedCache
from rows_world import BF16, D, World
from test_gpu_rows import check_rows, check_token

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load_library()


def handle(c):
    ones = torch.ones((c.S, 7))
    return MemDecay(c, ones, ones * 0.01, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0)


@pytest.mark.parametrize("P", [16, 64])
def test_bounds_behind_a_chunk(P):
    """Of every page, as if the keys had been loaded at once."""
    kw = dict(L=2, Hq=4, Hkv=2, d=D, P=P, S=2, max_pages=20, n_phys=40, values="e4m3", bounds=True)
    one, two = PagedCache(**kw), PagedCache(**kw)
    keys = torch.randn((300, 2, 2, D), generator=torch.Generator().manual_seed(1)).to(BF16).to(one.device)
    m = PagedCache.pages_for([1] * 300, P, False)
    one.load_session(0, keys, [1] * 300, list(range(m)), budget=300, clock=300)
    first = PagedCache.pages_for([1] * 100, P, False)
    two.load_session(0, keys[:100], [1] * 100, list(range(first)), budget=300, clock=100)
    two.load_values(0, keys[:100])
    two.set_free_pages(list(range(39, first - 1, -1)))
    a, b = handle(one), handle(two)
    a.update_bounds(True)
    b.update_bounds(True)
    at = two.place_tokens(0, [1] * 200)
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32, device=two.device)
    for layer in range(2):
        b.write_rows(layer, i32([0, 200, 200]), keys[100:, layer], keys[100:, layer], row_slot=i32(at))
    b.update_bounds(True)
    assert a.device_status() == 0 and b.device_status() == 0
    assert two.page_table[0, :m].tolist() == list(range(m))
    assert torch.equal(one.key_bounds[:m], two.key_bounds[:m]) and torch.equal(one.bound_exp[:m], two.bound_exp[:m])
    q = torch.randn((2, 4, D), device=two.device)
    lists = []
    for md in (a, b):
        blocks, count = torch.zeros((2, 2, 4), dtype=torch.int32, device=two.device), torch.zeros((2, 2), dtype=torch.int32, device=two.device)
        md.select_blocks(1, q, blocks, count)
        lists.append((blocks, count))
    assert torch.equal(lists[0][0], lists[1][0]) and torch.equal(lists[0][1], lists[1][1])


@pytest.mark.parametrize("aligned", [False, True])
def test_windows_count_slots_of_the_cache_as_it_stands(aligned):
    """Before and behind an eviction, holes among them."""
    w = World(1, 4, 2, 16, [150, 90], seed=261, aligned=aligned, spare=10, extra=10)
    w.md.observe(0, w.normal(2, 1, 1, 4, D))
    w.md.score()
    serials = [w.cache.page_serial[s, :int(w.cache.n_pages[s])].tolist() for s in range(2)]
    gone = [[serials[0][i] for i in (0, 3, 4)], [serials[1][i] for i in (1, 2)]]
    lists = torch.zeros((2, w.cache.max_pages), dtype=torch.int32, device=w.dev)
    for s in range(2):
        lists[s, :len(gone[s])] = w.i32(gone[s])
    for turn in range(2):
        for kw in (dict(window=40, sinks=3), dict(window=20), dict(window=64, sinks=40)):
            q, out, lse = w.normal(2, 4, D), torch.empty((2, 4, D), device=w.dev), torch.empty((2, 4), device=w.dev)
            w.md.attend(0, q, out, lse=lse, **kw)
            check_token(w, 0, q, out, lse, None, None, **kw)
            start_d, slot_d, start, slot = w.rows([9, 4])
            q, out, lse = w.normal(13, 4, D), torch.empty((13, 4, D), device=w.dev), torch.empty((13, 4), device=w.dev)
            w.md.attend_rows(0, q, out, start_d, row_slot=slot_d, lse=lse, **kw)
            check_rows(w, 0, q, out, lse, start, slot, **kw)
        if turn == 0:
            w.md.compact(lists, w.i32([3, 2]))
            assert w.md.device_status() == 0
            for s in range(2):
                keep = ~np.isin(np.repeat(serials[s], 16)[:w.slots[s]], gone[s])
                w.k[s], w.v[s] = (x[s][torch.as_tensor(keep)] for x in (w.k, w.v))
                w.live[s], w.slots[s] = w.live[s][keep], int(keep.sum())
                assert int(w.cache.n_tokens[s]) == w.slots[s]
