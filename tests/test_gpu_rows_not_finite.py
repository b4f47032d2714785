"""Values that are not finite among a prompt's: each row has them in the very
dims in which it sees one, the other dims and rows are as without them, and
rows that see them all alike take the time of any others."""
import math

import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import PagedCache
from rows_world import BF16, D, World, attend, attention_bound, visible
from test_gpu_rows import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load_library()


def put(w, t, e, x):
    """Value x in dim e of the session's token t (all layers and KV heads)."""
    page, o = int(w.ids[0][t // w.P]), t % w.P
    if w.coded:   # a NaN code
        assert math.isnan(x)
        at = (o // 16, e // 64, o // 4 % 4, e % 16, e // 16 % 4, o % 4)
        w.cache.v_codes[(page, slice(None), slice(None)) + at] = 0x7F
    else:
        y = PagedCache.from_value_layout(w.cache.v_pool[page:page + 1]).contiguous()
        y[0, o, :, :, e] = x
        w.cache.v_pool[page:page + 1] = PagedCache.to_value_layout(y)
    w.v[0][t, ..., e] = x


def check(w, q, out, lse, slot, rows, **kw):
    rounded = q.dtype == BF16 and out.dtype == BF16
    qh, oh, lh = q.cpu(), out.cpu(), lse.cpu().double()
    for r in rows:
        seen = visible(w.live[0], slot[r], kw.get("window", 0), kw.get("sinks", 0))
        for kv in range(w.Hkv):
            k, v = w.k[0][:, 0, kv], w.v[0][:, 0, kv]
            hs = slice(kv * w.G, (kv + 1) * w.G)
            odd = ~v.isfinite() & seen[:, None]
            v0 = torch.where(v.isfinite(), v, 0.0)
            ref, rl, dev = attend(qh[r, hs].float(), k, v0, seen)
            tol, ltol = attention_bound(qh[r, hs].float(), k, v0, seen, dev, ref, rl, rounded, out.dtype)
            got, gl = oh[r, hs].double(), lh[r, hs]
            fine = ~odd.any(0)
            assert bool(got[:, fine].isfinite().all()) and not bool(got[:, ~fine].isfinite().any()), (r, slot[r], kv)
            assert bool(((got - ref).abs() <= tol)[:, fine].all()), (r, slot[r], kv)
            assert bool(((gl - rl).abs() <= ltol).all()), (r, slot[r], kv)
            for e in (~fine).nonzero()[:, 0].tolist():
                x = v[odd[:, e], e]
                if rounded and bool((x == math.inf).all()):   # (weights of several terms make NaN of it)
                    assert bool((got[:, e] == math.inf).all()), (r, slot[r], kv, e)


@pytest.mark.parametrize("types", TYPES, ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("n,heads", [(400, 16), (400, 2), (5, 4)], ids=["many", "some", "few"])
def test_each_row_has_what_it_sees(n, heads, coded, types):
    print("[not finite]", n, heads, coded, types, flush=True)
    w = World(1, heads, 1, 16, [700], seed=251, coded=coded, quant=0.4)
    for t, e, x in ((3, 7, math.inf), (310, 100, -math.inf), (450, 5, math.nan), (697, 66, math.inf), (690, 7, math.nan)):
        put(w, t, e, math.nan if coded else x)
    slot = np.arange(700 - n, 700)
    q = w.normal(n, heads, D).to(types[0])
    for kw in (dict(), dict(window=130, sinks=5), dict(window=40)):
        out, lse = torch.zeros((n, heads, D), dtype=types[1], device=w.dev), torch.zeros((n, heads), device=w.dev)
        w.md.attend_rows(0, q, out, w.i32([0, n]), lse=lse, **kw)
        rows = sorted(set(range(0, n, 37)) | set(range(max(0, n - 14), n)) | ({5, 9, 10, 11, 12, 149, 150, 151} if n == 400 else set()))
        check(w, q, out, lse, slot, rows, **kw)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("many", [True, False])
def test_scales_that_are_none_beside_scales_that_do_not_fit(many, types):
    w = World(1, 16, 1, 16, [300], seed=252)
    w.cache.v_scale[int(w.ids[0][2])] = math.nan
    w.v[0][32:48] = math.nan
    scale = w.cache.v_scale[int(w.ids[0][11])]
    before = scale.cpu().double()
    scale *= 2.0 ** 110
    w.v[0][176:192] *= scale.cpu().double() / before
    slot = np.arange(300) if many else np.array([5, 20, 40, 180, 250, 299])
    n = len(slot)
    q = w.normal(n, 16, D).to(types[0])
    for kw in (dict(), dict(window=120)):
        out, lse = torch.zeros((n, 16, D), dtype=types[1], device=w.dev), torch.zeros((n, 16), device=w.dev)
        w.md.attend_rows(0, q, out, w.i32([0, n]), row_slot=w.i32(slot), lse=lse, **kw)
        check(w, q, out, lse, slot, range(0, n, 7 if many else 1), **kw)


@pytest.mark.parametrize("coded", [True, False])
def test_rows_that_see_one_take_no_longer(coded):
    """One in the first token, which 2,048 rows of 16 heads see: a time of the
    order of theirs without it (summed again one by one they took hundreds of
    times as long)."""
    w = World(1, 16, 1, 16, [2048], seed=253, coded=coded)
    q = w.normal(2048, 16, D).to(BF16)
    out, lse = torch.zeros_like(q), torch.zeros((2048, 16), device=w.dev)
    start = w.i32([0, 2048])

    def time():
        got = []
        for _ in range(7):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in "ab")
            a.record()
            w.md.attend_rows(0, q, out, start, lse=lse)
            b.record()
            torch.cuda.synchronize()
            got.append(a.elapsed_time(b))
        return sorted(got)[3]

    without = time()
    if coded:
        w.cache.v_scale[int(w.ids[0][0])] = math.nan
        w.v[0][:16] = math.nan
    else:
        put(w, 0, 9, math.inf)
    one = time()
    print("[not finite] us without, with:", without * 1e3, one * 1e3, flush=True)
    check(w, q, out, lse, np.arange(2048), range(0, 2048, 211))
    assert one < 10 * without
