"""Rows whose slot is not the session's, among rows that are there: the
attention gives them zeros and a log sum of -infinity, whatever their
neighbours see, and the neighbours' results are those of a call without them."""
import math

import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import PagedCache
from rows_world import BF16, D, World
from test_gpu_rows import TYPES, check_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load_library()


def run_absent(w, counts, absent, types, seed=0, **kw):
    """Late rows of each session, `absent` of which are not there."""
    rng = np.random.default_rng(seed)
    start = np.concatenate([[0], np.cumsum(counts)])
    slot, there = [], []
    for s, n in enumerate(counts):
        mine = np.sort(rng.choice(np.arange(w.slots[s] // 2, w.slots[s]), n, replace=n > w.slots[s] // 2))
        gone = rng.random(n) < absent
        gone[:1] = True
        mine[gone] = rng.choice([-1, -1, w.slots[s], w.slots[s] + 7, 2 ** 31 - 1, -2 ** 31], int(gone.sum()))
        slot += mine.tolist()
        there += (~gone).tolist()
    n = len(slot)
    q = w.normal(n, w.Hq, D).mul(1.5).to(types[0])
    out = torch.full((n, w.Hq, D), 5.0, dtype=types[1], device=w.dev)
    lse = torch.full((n, w.Hq), 5.0, device=w.dev)
    w.md.attend_rows(0, q, out, w.i32(start), row_slot=w.i32(slot), lse=lse, **kw)
    torch.cuda.synchronize()
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    there = np.array(there)
    gone = torch.as_tensor(np.flatnonzero(~there), device=w.dev)
    assert bool((out[gone] == 0).all()) and bool((lse[gone] == -math.inf).all())
    rows = np.flatnonzero(there)
    check_rows(w, 0, q, out, lse, start, np.array(slot), some=rows[:: max(1, len(rows) // 25)].tolist(), **kw)


KW = [dict(), dict(window=90, sinks=20)]


@pytest.mark.parametrize("types", TYPES, ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("lens,counts", [([100], [2]), ([300, 40], [9, 5]), ([9000, 500], [6, 30])], ids=["short", "two", "parts"])
def test_few_rows_some_not_there(lens, counts, coded, types):
    print("[absent few]", lens, coded, types, flush=True)
    w = World(1, 4, 2, 16, lens, seed=201, coded=coded)
    for kw in KW:
        run_absent(w, counts, 0.5, types, seed=len(lens), **kw)


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("lens,counts", [([300, 40], [160, 20]), ([5000, 700], [200, 60])], ids=["short", "parts"])
@pytest.mark.parametrize("absent", [0.02, 0.9])
def test_many_rows_some_not_there(absent, lens, counts, coded):
    print("[absent many]", absent, lens, coded, flush=True)
    w = World(1, 16, 1, 16, lens, seed=202, coded=coded)
    for kw in KW:
        run_absent(w, counts, absent, TYPES[0], seed=3, **kw)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("many", [True, False])
def test_values_that_are_not_finite_beside_rows_that_are_not_there(many, types):
    """A block that holds an infinity and that every row there sees in full:
    these are infinite in its dimension, those not there still zero."""
    w = World(1, 16, 1, 16, [400], seed=203, coded=False)
    page = int(w.ids[0][2])
    y = PagedCache.from_value_layout(w.cache.v_pool[page:page + 1]).contiguous()
    y[0, 3, 0, 0, 9] = math.inf
    w.cache.v_pool[page:page + 1] = PagedCache.to_value_layout(y)
    n = 150 if many else 4
    slot = np.arange(390 - n, 390)
    slot[::3] = -1
    q = w.normal(n, 16, D).to(types[0])
    out, lse = torch.full((n, 16, D), 5.0, dtype=types[1], device=w.dev), torch.full((n, 16), 5.0, device=w.dev)
    w.md.attend_rows(0, q, out, w.i32([0, n]), row_slot=w.i32(slot), lse=lse)
    assert bool((out[::3] == 0).all()) and bool((lse[::3] == -math.inf).all())
    there = torch.as_tensor(slot >= 0, device=w.dev)
    assert not bool(out[there][..., 9].isfinite().any())
    assert bool(out[there][..., :9].isfinite().all()) and bool(out[there][..., 10:].isfinite().all())


def test_only_rows_that_are_not_there():
    w = World(1, 16, 1, 16, [400], seed=204)
    for n, types in ((3, TYPES[0]), (3, TYPES[1]), (200, TYPES[0])):
        q = w.normal(n, 16, D).to(types[0])
        out, lse = torch.full((n, 16, D), 5.0, dtype=types[1], device=w.dev), torch.full((n, 16), 5.0, device=w.dev)
        w.md.attend_rows(0, q, out, w.i32([0, n]), row_slot=w.i32([-1] * n), lse=lse, window=7)
        assert w.md.device_status() == B.MD_DEV_BAD_ROW
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
