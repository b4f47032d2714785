"""Rows written among others whose slots are not the session's (-1, or past its
tokens), wherever these lie: the cache holds what a call without them leaves."""
import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import PagedCache
from rows_world import BF16, D, World, quantise_slots
from test_gpu_rows import check_written, kv_rows, pool_slots, same

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load_library()


NONE = np.array([-1, -1, -1, -2 ** 31, 2 ** 31 - 1, 10 ** 6])


def padded(rng, slots, where):
    """The slots of a session's rows among others that are not there."""
    none = lambda n: rng.choice(NONE, n)
    n = len(slots)
    if where == "front":
        return np.concatenate([none(rng.integers(1, 6)), slots])
    if where == "behind":
        return np.concatenate([slots, none(rng.integers(1, 6))])
    if where == "far behind":
        return np.concatenate([slots, none(700)])
    if where == "far in front":
        return np.concatenate([none(700), slots])
    if where == "fixed":      # every session's rows in a place of 64
        return np.concatenate([slots, none(-n % 64)])
    out = []                  # between: now and then some, or many
    for t in slots:
        out.append(t)
        if rng.random() < 0.2:
            out += none(rng.choice([1, 2, 40])).tolist()
    return np.array(out, dtype=int)


WHERE = ["front", "behind", "far behind", "far in front", "fixed", "between"]


@pytest.mark.parametrize("where", WHERE)
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("chunk,P,aligned", [(1000, 16, False), (7, 16, False), (19, 64, True)])
def test_rows_that_are_not_there_leave_the_others(chunk, P, aligned, coded, where):
    print("[padded]", chunk, P, aligned, coded, where, flush=True)
    lens = [700, 0, 1, 16, 17, 259] if chunk > 19 else [45, 0, 1, 16, 17, 30]
    w = World(1, 4, 2, P, lens, seed=211, coded=coded, aligned=aligned, fill=False)
    rng = np.random.default_rng(5)
    done = np.zeros(w.S, dtype=int)
    while (done < np.array(lens)).any():
        step = np.minimum(chunk, np.array(lens) - done)
        lists, real = [], []
        for s in range(w.S):
            mine = np.flatnonzero(w.live[s])[done[s]:done[s] + step[s]]
            lists.append(padded(rng, mine, where))
        start = np.concatenate([[0], np.cumsum([len(x) for x in lists])])
        slot = np.concatenate(lists).astype(int)
        there = np.concatenate([(x >= 0) & (x < w.slots[s]) for s, x in enumerate(lists)])
        own = np.concatenate([[0], np.cumsum(step)])
        k, v = (torch.full((len(slot), w.Hkv, D), 9.0, dtype=BF16, device=w.dev) for _ in "kv")
        at = torch.as_tensor(np.flatnonzero(there), device=w.dev)
        rows = kv_rows(w, own, slot[there], 0)
        k[at], v[at] = rows[0], rows[1]
        w.md.write_rows(0, w.i32(start), k, v, row_slot=w.i32(slot))
        assert w.md.device_status() == (0 if there.all() else B.MD_DEV_BAD_ROW)
        done += step
    check_written(w, [0])


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("where", ["behind", "front", "between"])
def test_long_prompts_in_longer_places(where, coded):
    """Searches over thousands of rows that are not there."""
    print("[padded long]", where, coded, flush=True)
    n, place = 3000, 9000
    w = World(1, 1, 1, 16, [n], seed=212, coded=coded, fill=False)
    slot = np.full(place, -1)
    at = {"behind": np.arange(n), "front": np.arange(place - n, place),
          "between": np.sort(np.random.default_rng(1).choice(place, n, replace=False))}[where]
    slot[at] = np.arange(n)
    rows = kv_rows(w, np.array([0, n]), np.arange(n), 0)
    k, v = (torch.full((place, 1, D), 9.0, dtype=BF16, device=w.dev) for _ in "kv")
    at = torch.as_tensor(at, device=w.dev)
    k[at], v[at] = rows[0], rows[1]
    w.md.write_rows(0, w.i32([0, place]), k, v, row_slot=w.i32(slot))
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    check_written(w, [0])


def test_more_rows_than_tokens_without_slots():
    """Without slots the rows are the session's last ones; those too many are not there."""
    for coded in (True, False):
        w = World(1, 1, 1, 16, [20, 5], seed=213, coded=coded, fill=False)
        rows = kv_rows(w, np.array([0, 20, 25]), np.concatenate([np.arange(20), np.arange(5)]), 0)
        none = torch.full((21, 1, D), 9.0, dtype=BF16, device=w.dev)
        k, v = (torch.cat([none, x[:20], none[:2], x[20:]]) for x in rows)
        w.md.write_rows(0, w.i32([0, 41, 48]), k, v)
        assert w.md.device_status() == B.MD_DEV_BAD_ROW
        check_written(w, [0])


def test_which_rows_count():
    """Rows that are not there do not stand in the way of those around them, a
    row that is not above those before it is left out."""
    w = World(1, 1, 1, 16, [40, 40], seed=214, coded=False, fill=False)
    slot = [-1, 5, 6, 6, 40, 3, 8, 2 ** 31 - 1, -2 ** 31] + [-1, 17, -1, 20, 20, 50, 33]
    k = torch.arange(16, device=w.dev, dtype=torch.float32)[:, None, None].expand(16, 1, D).to(BF16).contiguous()
    w.md.write_rows(0, w.i32([0, 9, 16]), k, k, row_slot=w.i32(slot))
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    for s, want in ((0, {5: 1, 6: 2, 8: 6}), (1, {17: 10, 20: 12, 33: 15})):
        for got in pool_slots(w, s):
            have = {int(t): int(got[t, 0, 0, 0]) for t in (~got[:, 0, 0, 0].isnan()).nonzero()}
            assert have == want, (s, have)


def test_a_row_in_front_that_is_not_there_in_the_middle_of_a_block():
    """The rows behind it go on in the open block, whose tokens stay."""
    w = World(1, 2, 2, 16, [30], seed=215, fill=False)
    for lo, hi, front, behind in ((0, 5, 0, 3), (5, 7, 2, 1), (7, 21, 1, 2), (21, 30, 3, 0)):
        slot = np.concatenate([np.full(front, -1), np.arange(lo, hi), np.full(behind, -1)])
        rows = kv_rows(w, np.array([0, hi - lo]), np.arange(lo, hi), 0)
        k, v = (torch.cat([torch.full((front, 2, D), 9.0, dtype=BF16, device=w.dev), x,
                           torch.full((behind, 2, D), 9.0, dtype=BF16, device=w.dev)]) for x in rows)
        w.md.write_rows(0, w.i32([0, len(slot)]), k, v, row_slot=w.i32(slot))
    check_written(w, [0])


@pytest.mark.parametrize("coded", [True, False])
def test_a_key_for_a_page_of_codes_is_left_out_and_its_value_written(coded):
    w = World(1, 2, 2, 16, [70], seed=216, quant=1.0, coded=coded)
    keys = w.cache.k_pool.clone()
    pages = w.cache.page_format.bool()
    assert int(pages.sum()) == 4
    k, v = (w.normal(70, 2, D, dtype=BF16) for _ in "kv")
    w.md.write_rows(0, w.i32([0, 70]), k, v)
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    assert torch.equal(keys[pages].view(torch.uint8), w.cache.k_pool[pages].view(torch.uint8))
    last = torch.as_tensor(w.ids[0][4:], device=w.dev)
    assert torch.equal(PagedCache.from_pool_layout(w.cache.k_pool[last])[0, :6, 0], k[64:])
    want = v.float().cpu()
    if coded:
        want = quantise_slots(want).float()
        assert same(w.cache.v_open[0, 0, :, :6], v[64:].transpose(0, 1))
    assert same(pool_slots(w, 0)[1][:70, 0], want)
    w.md.write_rows(0, w.i32([0, 70]), v=v)
    assert w.md.device_status() == 0
