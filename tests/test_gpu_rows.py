"""Rows into, out of and over the paged cache, and 8-bit values, on the device
against 64-bit definitions.

What is moved or quantised is equal, bit for bit: a code is the E4M3 value
nearest to the float32 quotient, which IEEE division defines.  The attention's
tolerances are derived in rows_world.attention_bound."""
import math

import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import MemDecay, PagedCache
from rows_world import BF16, D, World, attend, attention_bound, quantise_slots, visible

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load_library()


def say(*a):
    print(*a, flush=True)


def same(a, b):
    """Equal bits where neither is NaN, and NaN in the same places."""
    a, b = a.double().cpu(), b.double().cpu()
    return a.shape == b.shape and torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))


# ---------------------------------------------------------------- writing

def pool_slots(w, s):
    """What the pools hold for a session's slots: keys, values [slots][L][Hkv][d] float64."""
    c = w.cache
    ids = torch.as_tensor(w.ids[s], device=w.dev)
    k = PagedCache.from_pool_layout(c.k_pool[ids]).flatten(0, 1)
    v = PagedCache.from_code_layout(c.v_codes[ids], c.v_scale[ids]) if w.coded else PagedCache.from_value_layout(c.v_pool[ids])
    return k.double().cpu(), v.flatten(0, 1).double().cpu()


def check_written(w, layers, upto=None):
    for s in range(w.S):
        if w.slots[s] == 0:
            continue
        k, v = pool_slots(w, s)
        n = w.slots[s]
        live = torch.as_tensor(w.live[s])
        want_v = w.v[s]
        for l in layers:
            assert same(k[:n, l][live], w.k[s][:, l][live]), ("keys", s, l)
            assert same(v[:n, l][live], want_v[:, l][live].float()), ("values", s, l)
            dead = torch.ones(len(k), dtype=torch.bool)
            dead[:n] = ~live
            assert k[dead][:, l].isnan().all(), ("other slots' keys", s, l)
            if not w.coded:
                assert v[dead][:, l].isnan().all(), ("other slots' values", s, l)
        for l in set(range(w.L)) - set(layers):
            assert k[:, l].isnan().all() and v[:, l].isnan().all(), ("other layers", s, l)
        if w.coded:
            last = (n - 1) // 16 * 16
            tail = torch.zeros(16, w.L, w.Hkv, D)
            tail[:n - last] = w.v16[s][last:n]
            for l in layers:
                assert same(w.cache.v_open[s, l], tail[:, l].permute(1, 0, 2)), ("open block", s, l)


def kv_rows(w, start, slot, layer, pad=0):
    """Key and value rows of the listed slots, as a part of wider rows."""
    n = int(start[-1])
    both = torch.full((n + 2, 2, w.Hkv, D + pad), math.nan, dtype=BF16, device=w.dev)[:n, ..., :D] if pad == 0 else None
    if pad:
        wide = torch.full((n, 2 * w.Hkv * D + pad), math.nan, dtype=BF16, device=w.dev)
        both = wide[:, :2 * w.Hkv * D].view(n, 2, w.Hkv, D)
    session = np.repeat(np.arange(w.S), np.diff(start))
    for i, x in enumerate((w.k, w.v16)):
        if n:
            both[:, i] = torch.stack([x[s][t, layer] for s, t in zip(session, slot)]).to(BF16).to(w.dev)
    return both[:, 0], both[:, 1]


LENS = [700, 0, 1, 16, 17, 259]


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("aligned", [False, True])
@pytest.mark.parametrize("shape", [(2, 12, 2), (1, 5, 5), (1, 4, 1)])
@pytest.mark.parametrize("chunk", [1000, 7])
def test_written_rows(chunk, shape, aligned, coded, P):
    say("[write]", chunk, shape, aligned, coded, P)
    lens = LENS if chunk > 7 else [45, 0, 1, 16, 17, 30]
    w = World(*shape, P, lens, seed=11, coded=coded, aligned=aligned, fill=False)
    layer = w.L - 1
    done = np.zeros(w.S, dtype=int)
    while (done < np.array(lens)).any():
        step = np.minimum(chunk, np.array(lens) - done)
        first = [int(np.flatnonzero(w.live[s])[done[s]]) if step[s] else w.slots[s] for s in range(w.S)]
        start_d, slot_d, start, slot = w.rows(step, first)
        k, v = kv_rows(w, start, slot, layer, pad=8 if chunk > 7 else 0)
        w.md.write_rows(layer, start_d, k, v, row_slot=slot_d)
        done += step
    assert w.md.device_status() == 0
    check_written(w, [layer])


@pytest.mark.parametrize("coded", [True, False])
def test_rows_without_slots_are_the_last_ones(coded):
    w = World(1, 2, 2, 16, [33, 0, 5], seed=12, coded=coded, fill=False)
    start_d, _, start, slot = w.rows([33, 0, 5])
    k, v = kv_rows(w, start, slot, 0)
    w.md.write_rows(0, start_d, k, v)
    assert w.md.device_status() == 0
    check_written(w, [0])
    # keys alone and values alone
    u = World(1, 2, 2, 16, [33, 0, 5], seed=12, coded=coded, fill=False)
    u.md.write_rows(0, start_d, k)
    assert PagedCache.from_pool_layout(u.cache.k_pool).isfinite().any()
    assert (u.cache.v_scale if coded else u.cache.v_pool).isnan().all()
    u.md.write_rows(0, start_d, v=v)
    check_written(u, [0])


def test_rows_behind_the_last_session_and_other_pages_are_left_alone():
    w = World(1, 3, 3, 16, [20, 40], seed=13, fill=False)
    start_d, slot_d, start, slot = w.rows([20, 40])
    k, v = kv_rows(w, start, slot, 0)
    more = torch.full((50, 3, D), 9.0, dtype=BF16, device=w.dev)
    w.md.write_rows(0, start_d, torch.cat([k, more]), torch.cat([v, more]),
                    row_slot=torch.cat([slot_d, torch.zeros(50, dtype=torch.int32, device=w.dev)]))
    assert w.md.device_status() == 0
    check_written(w, [0])
    others = np.setdiff1d(np.arange(w.cache.n_phys), np.concatenate(w.ids))
    assert w.cache.k_pool[torch.as_tensor(others, device=w.dev)].isnan().all()
    assert (w.cache.v_codes[torch.as_tensor(others, device=w.dev)] == 0x7F).all()


@pytest.mark.parametrize("S", [65, 1024])
def test_many_sessions_written_and_read(S):
    lens = [(5 * s) % 37 for s in range(S)]
    w = World(1, 1, 1, 16, lens, seed=14, fill=False)
    start_d, slot_d, start, slot = w.rows(lens)
    k, v = kv_rows(w, start, slot, 0)
    w.md.write_rows(0, start_d, k, v)
    assert w.md.device_status() == 0
    check_written(w, [0])
    ko, vo = torch.empty_like(k, memory_format=torch.contiguous_format), torch.empty((len(slot), 1, D), device=w.dev, dtype=BF16)
    w.md.read_rows(0, start_d, ko, vo)
    assert torch.equal(ko, k)


def test_unusual_values():
    """Zero blocks, the least and the largest values, and blocks with a value that is not finite."""
    w = World(1, 1, 1, 16, [16 * 6], seed=15, fill=False)
    v = w.v16[0]
    v[0:16] = 0.0
    v[16:32] = 2.0 ** -126
    v[32:48] = 3.3895e38
    v[50, 0, 0, 3] = math.inf
    v[70, 0, 0, 5] = math.nan
    v[80:96] = torch.randn(16, 1, 1, D, generator=w.g) * 2.0 ** -100
    v.copy_(v.to(BF16).float())
    w.v[0] = quantise_slots(v.flatten(1, 2)).view(96, 1, 1, D)
    start_d, slot_d, start, slot = w.rows([96])
    k, vv = kv_rows(w, start, slot, 0)
    w.md.write_rows(0, start_d, k, vv)
    check_written(w, [0])
    got = pool_slots(w, 0)[1]
    assert got[48:64].isnan().all() and got[64:80].isnan().all() and torch.equal(got[:16], torch.zeros(16, 1, 1, D).double())
    # (all of a block alike: every one is the top code; its scale's quotient and product round once each)
    assert ((got[32:48] - v[32:48]).abs() <= 2.0 ** -23 * v[32:48]).all()


def test_rows_that_do_not_count():
    """Slots outside the session, slots that do not ascend, the same slot
    twice: left out, and told of; the others arrive."""
    w = World(1, 1, 1, 16, [40, 40], seed=16, coded=False, fill=False)
    slot = [-1, 5, 6, 6, 40, 3, 8, 2 ** 31 - 1, -2 ** 31] + [0, 17, 20, 18, 33]
    start = [0, 9, 14]
    want = {(0, 5), (0, 6), (0, 8), (1, 0), (1, 17), (1, 20), (1, 33)}
    k = torch.arange(14, device=w.dev, dtype=torch.float32)[:, None, None].expand(14, 1, D).to(BF16).contiguous()
    w.md.write_rows(0, w.i32(start), k, k, row_slot=w.i32(slot))
    assert w.md.device_status() & B.MD_DEV_BAD_ROW
    for s in range(2):
        got, vals = pool_slots(w, s)
        have = {int(t) for t in (~got[:, 0, 0, 0].isnan()).nonzero()}
        assert have <= {t for z, t in want if z == s} and torch.equal(got.nan_to_num(-1), vals.nan_to_num(-1))
    assert int((~pool_slots(w, 1)[0][:, 0, 0, 0].isnan()).sum()) == 4


def test_row_starts_that_do_not_ascend():
    """Nobody's rows: nothing is written, read or attended."""
    w = World(1, 1, 1, 16, [40, 40, 40], seed=16, coded=False, fill=False)
    before = w.cache.k_pool.clone()
    k, v = (torch.full((14, 1, D), 5.0, dtype=BF16, device=w.dev) for _ in "kv")
    for bad in ([0, 9, 5, 14], [3, 14, 15, 15], [-4, 2, 14, 14], [0, -1, 14, 14], [0, 14, 0, 14], [14, 0, 14, 0], [0, 0, 2 ** 31 - 1, 3]):
        for types in ((torch.float32, torch.float32), (BF16, BF16)):
            w.md.write_rows(0, w.i32(bad), k, v, row_slot=w.i32(list(range(14))))
            assert w.md.device_status() == B.MD_DEV_BAD_ROW, bad
            out = torch.full((14, 1, D), 5.0, dtype=types[1], device=w.dev)
            w.md.attend_rows(0, torch.zeros((14, 1, D), dtype=types[0], device=w.dev), out, w.i32(bad), row_slot=w.i32([0] * 14))
            assert w.md.device_status() == B.MD_DEV_BAD_ROW, bad
            assert (out == 5).all()
            w.md.read_rows(0, w.i32(bad), k, v, row_slot=w.i32([0] * 14))
            assert w.md.device_status() == B.MD_DEV_BAD_ROW and (k == 5).all() and (v == 5).all()
    assert torch.equal(before.view(torch.uint8), w.cache.k_pool.view(torch.uint8))


def test_descending_lists_give_the_same_bits_every_time():
    """A list that breaks its rule writes each block at most once."""
    first = None
    for _ in range(3):
        w = World(1, 2, 2, 16, [64], seed=17, fill=False)
        slot = [20, 3, 21, 4, 22, 5, 60, 17, 18, 33, 2, 19]
        g = torch.Generator().manual_seed(3)
        k = torch.randn((12, 2, D), generator=g).to(BF16).to(w.dev)
        w.md.write_rows(0, w.i32([0, 12]), k, k, row_slot=w.i32(slot))
        assert w.md.device_status() == B.MD_DEV_BAD_ROW
        bits = (w.cache.v_codes.clone(), w.cache.v_scale.clone(), w.cache.k_pool.clone(), w.cache.v_open.clone())
        if first is None:
            first = bits
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, bits))


def test_pages_of_codes_keep_their_keys():
    w = World(1, 2, 2, 16, [64], seed=18, quant=1.0)
    before = w.cache.k_pool.clone()
    assert w.cache.page_format.sum() > 0
    start_d, slot_d, start, slot = w.rows([64])
    k, v = kv_rows(w, start, slot, 0)
    w.md.write_rows(0, start_d, (-k).contiguous(), v.contiguous())
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    coded = w.cache.page_format.bool()
    assert torch.equal(before[coded].view(torch.uint8), w.cache.k_pool[coded].view(torch.uint8))
    w.md.write_rows(0, start_d, v=v)   # values go there
    assert w.md.device_status() == 0
    live_v = pool_slots(w, 0)[1][:64]
    assert same(live_v, w.v[0].float())


# ---------------------------------------------------------------- the step's values

@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("aligned", [False, True])
def test_appended_values_are_those_of_whole_blocks(aligned, P):
    say("[append]", aligned, P)
    w = World(2, 4, 2, P, [0, 1, 15, 16, 40, 70], seed=21, aligned=aligned, spare=40, extra=40)
    w.md.observe(0, None)
    for step in range(1, 40):
        big = 4.0 if step % 7 == 3 else 1.0        # now and then the scale grows
        nk, nv = (w.normal(w.S, 2, 2, D) for _ in range(2))
        nv = (nv * big).to(BF16)
        region = w.rng.integers(0, 7, w.S) if step % 5 == 0 else np.zeros(w.S, dtype=int)
        w.md.observe(step, None, nk.to(BF16), torch.as_tensor(region.astype(np.uint8), device=w.dev))
        w.md.append_values(nv)
        assert w.md.device_status() == 0
        n = w.cache.n_tokens.tolist()
        for s in range(w.S):
            old = len(w.v16[s])
            v = torch.zeros((n[s], 2, 2, D))
            v[:old] = w.v16[s]
            v[-1] = nv[s].float().cpu()
            w.v16[s] = v
            w.live[s] = np.concatenate([w.live[s], np.zeros(n[s] - old, bool)])
            w.live[s][-1] = True
            w.slots[s] = n[s]
        if step in (1, 2, 17, 39):
            for s in range(w.S):
                m = -(-n[s] // P)
                ids = w.cache.page_table[s, :m].long()
                got = PagedCache.from_code_layout(w.cache.v_codes[ids], w.cache.v_scale[ids]).flatten(0, 1)[:n[s]]
                want = quantise_slots(w.v16[s].flatten(1, 2)).view(n[s], 2, 2, D)
                live = torch.as_tensor(w.live[s])
                assert same(got[live.to(w.dev)], want[live].float()), (s, step)
                o = (n[s] - 1) % 16
                assert same(w.cache.v_open[s, :, :, :o + 1].permute(2, 0, 1, 3), w.v16[s][n[s] - 1 - o:])


def test_values_that_are_not_finite_when_appended():
    w = World(1, 1, 1, 16, [3], seed=22)
    w.md.observe(0, None)
    for step, x in enumerate([1.0, math.inf, 2.0], start=1):
        w.md.observe(step, None, w.normal(1, 1, 1, D, dtype=BF16), torch.zeros(1, dtype=torch.uint8, device=w.dev))
        w.md.append_values(torch.full((1, 1, 1, D), x, dtype=BF16, device=w.dev))
        page = int(w.cache.page_table[0, 0])
        assert bool(w.cache.v_scale[page].isnan().all()) == (step > 1)


def test_appending_needs_a_step():
    w = World(1, 1, 1, 16, [3], seed=23)
    v = torch.zeros((1, 1, 1, D), dtype=BF16, device=w.dev)
    with pytest.raises(B.MemDecayError) as e:
        w.md.append_values(v)
    assert e.value.status == B.MD_E_STATE
    with pytest.raises(ValueError):
        w.md.append_values(v.float())


# ---------------------------------------------------------------- reading

@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("coded,quant,aligned", [(True, 0.0, False), (False, 0.0, True), (True, 0.6, False), (False, 0.6, True)])
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_read_rows(dtype, coded, quant, aligned, P):
    say("[read]", dtype, coded, quant, aligned, P)
    w = World(2, 6, 3, P, [300, 0, 1, 33, 16], seed=31, coded=coded, quant=quant, aligned=aligned)
    counts = [200, 0, 3, 40, 16]
    slot = np.concatenate([w.rng.choice(np.flatnonzero(w.live[s]), n) if n else np.zeros(0, int) for s, n in enumerate(counts)])
    slot[30:90] = np.flatnonzero(w.live[0])[10:70]         # a run of a session's rows
    start = np.concatenate([[0], np.cumsum(counts)])
    session = np.repeat(np.arange(w.S), counts)
    out = torch.full((len(slot) + 3, 2, 3, D), 5.0, dtype=dtype, device=w.dev)
    for layer in range(2):
        w.md.read_rows(layer, w.i32(start), out[:-3, 0], out[:-3, 1], row_slot=w.i32(slot))
        assert w.md.device_status() == 0
        for i, x in enumerate((w.k, w.v)):
            want = torch.stack([x[s][t, layer] for s, t in zip(session, slot)])
            # one float32 product, then bf16 (both round to nearest)
            want = want.float().to(dtype)
            assert torch.equal(out[:-3, i].cpu(), want), i
        assert (out[-3:] == 5.0).all()
    one = torch.full((int(start[-1]), 3, D), 5.0, dtype=dtype, device=w.dev)
    w.md.read_rows(1, w.i32(start), v_out=one, row_slot=w.i32(slot))
    assert torch.equal(one, out[:-3, 1])
    w.md.read_rows(1, w.i32(start), one, row_slot=w.i32(slot))
    assert torch.equal(one, out[:-3, 0])


def test_read_rows_that_are_not_there():
    w = World(1, 1, 1, 16, [20, 5], seed=32)
    k, v = (torch.full((8, 1, D), 5.0, device=w.dev) for _ in range(2))
    w.md.read_rows(0, w.i32([1, 4, 6]), k, v, row_slot=w.i32([0, 0, -1, 20, 5, 4, 0, 0]))
    assert w.md.device_status() == B.MD_DEV_BAD_ROW
    zero = [bool((k[i] == 0).all() and (v[i] == 0).all()) for i in range(8)]
    left = [bool((k[i] == 5).all() and (v[i] == 5).all()) for i in range(8)]
    assert zero == [False, False, True, True, True, False, False, False] and left == [True] + [False] * 5 + [True, True]


# ---------------------------------------------------------------- one token

def check_token(w, layer, q, out, lse, nk, nv, window=0, sinks=0, lists=None):
    q, out, lse = q.cpu(), out.cpu(), lse.cpu().double()
    for s in range(w.S):
        for kv in range(w.Hkv):
            k, v, live = w.k[s][:, layer, kv], w.v[s][:, layer, kv], w.live[s]
            if lists is not None:
                live = live & np.isin(np.arange(len(live)) // w.P, lists[s][kv])
            own = len(live) - 1
            if nk is not None:
                k = torch.cat([k, nk[s, kv].cpu().double()[None]])
                v = torch.cat([v, nv[s, kv].cpu().double()[None]])
                live = np.concatenate([live, [True]])
                own += 1
            seen = visible(live, own, window, sinks)
            qq = q[s, kv * w.G:(kv + 1) * w.G]
            ref, rl, dev = attend(qq, k, v, seen)
            got, gl = out[s, kv * w.G:(kv + 1) * w.G].double(), lse[s, kv * w.G:(kv + 1) * w.G]
            tol, ltol = attention_bound(qq, k, v, seen, dev, ref, rl, False, out.dtype)
            if not bool(seen.any()):
                assert torch.equal(got, ref) and torch.equal(gl, rl), (s, kv)
                continue
            assert bool(((got - ref).abs() <= tol).all()), (s, kv, float(((got - ref).abs() - tol).max()))
            assert bool(((gl - rl).abs() <= ltol).all()), (s, kv)


def run_token(w, layer=None, new=True, out_type=torch.float32, lists=None, **kw):
    layer = w.L - 1 if layer is None else layer
    q = w.normal(w.S, w.Hq, D) * 2
    nk, nv = (w.normal(w.S, w.Hkv, D, dtype=BF16) for _ in range(2)) if new else (None, None)
    out = torch.full((w.S, w.Hq, D), math.nan, dtype=out_type, device=w.dev)
    lse = torch.full((w.S, w.Hq), math.nan, device=w.dev)
    more = dict(kw)
    if lists is not None:
        most = max(1, max(len(x) for r in lists for x in r))
        b = torch.full((w.S, w.Hkv, most), -7, dtype=torch.int32)
        n = torch.zeros((w.S, w.Hkv), dtype=torch.int32)
        for s in range(w.S):
            for kv in range(w.Hkv):
                b[s, kv, :len(lists[s][kv])] = torch.tensor(lists[s][kv], dtype=torch.int32)
                n[s, kv] = len(lists[s][kv])
        more.update(blocks=b.to(w.dev), block_count=n.to(w.dev))
    w.md.attend(layer, q, out, new_k=nk, new_v=nv, lse=lse, **more)
    torch.cuda.synchronize()
    assert w.md.device_status() == 0
    check_token(w, layer, q, out, lse, nk, nv, lists=lists, **kw)


TOKEN_LENS = {"edges": [0, 1, 15, 16, 17, 31, 33, 63, 64, 65], "uneven": [1700, 3, 640, 0, 5000], "long": [20011]}


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("lens", sorted(TOKEN_LENS))
def test_token_over_codes(lens, new, P):
    say("[token]", lens, new, P)
    w = World(2, 12, 2, P, TOKEN_LENS[lens], seed=41)
    run_token(w, new=new)
    run_token(w, layer=0, new=new, out_type=BF16)


@pytest.mark.parametrize("shape", [(1, 1, 1), (3, 5, 5), (2, 16, 1), (1, 32, 8), (1, 14, 2)])
def test_token_head_layouts(shape):
    w = World(*shape, 16, [300, 0, 1, 2049], seed=42)
    run_token(w)
    run_token(w, out_type=BF16, new=False, window=100, sinks=3)


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("coded,aligned,quant", [(True, True, 0.0), (True, False, 0.6), (True, True, 0.6), (False, True, 0.6)])
def test_token_holes_and_codes(coded, aligned, quant, P):
    say("[token]", coded, aligned, quant, P)
    w = World(2, 12, 2, P, [700, 0, 1, 16, 2500], seed=43, coded=coded, aligned=aligned, quant=quant)
    run_token(w)
    run_token(w, new=False, window=130, sinks=20, out_type=BF16)
    lists = [[sorted(np.random.default_rng(s * 9 + kv).choice(len(w.ids[s]), min(len(w.ids[s]), 9), replace=False).tolist())
              if len(w.ids[s]) else [] for kv in range(w.Hkv)] for s in range(w.S)]
    run_token(w, lists=lists)


@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("new", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (16, 0), (17, 16), (33, 40), (640, 4), (5000, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_token_windows(window, sinks, new, coded):
    say("[window]", window, sinks, new, coded)
    w = World(1, 12, 2, 16 if coded else 64, [1700, 3, 640, 0, 16, 33, 31, 2600], seed=44, coded=coded)
    run_token(w, new=new, window=window, sinks=sinks)


def test_token_many_sessions():
    w = World(1, 2, 2, 16, [(7 * i) % 40 for i in range(1024)], seed=45)
    run_token(w)
    run_token(w, window=9, sinks=2)


def test_token_values_that_are_not_finite_outside_the_window():
    w = World(1, 2, 1, 16, [300], seed=46, coded=False)
    for t, x in ((3, math.inf), (200, math.nan), (281, -math.inf)):
        page = int(w.ids[0][t // 16])
        x_ = PagedCache.from_value_layout(w.cache.v_pool[page:page + 1]).contiguous()
        x_[0, t % 16] = x
        w.cache.v_pool[page:page + 1] = PagedCache.to_value_layout(x_)
        w.v[0][t] = x
    run_token(w, window=18, sinks=3, new=False)
    run_token(w, window=19, sinks=2)


# ---------------------------------------------------------------- ragged rows

def check_rows(w, layer, q, out, lse, start, slot, window=0, sinks=0, some=None, least=0.0):
    rounded = q.dtype == BF16 and out.dtype == BF16
    session = np.repeat(np.arange(w.S), np.diff(start))
    pick = range(len(slot)) if some is None else some
    qh, oh, lh = q.cpu(), out.cpu(), lse.cpu().double()
    for r in pick:
        s = session[r]
        seen = visible(w.live[s], slot[r], window, sinks)
        for kv in range(w.Hkv):
            k, v = w.k[s][:, layer, kv], w.v[s][:, layer, kv]
            hs = slice(kv * w.G, (kv + 1) * w.G)
            qq = qh[r, hs].float()
            ref, rl, dev = attend(qq, k, v, seen)
            got, gl = oh[r, hs].double(), lh[r, hs]
            tol, ltol = attention_bound(qq, k, v, seen, dev, ref, rl, rounded, out.dtype)
            if not bool(seen.any()):
                assert torch.equal(got, ref) and torch.equal(gl, rl), (r, kv)
                continue
            assert bool(((got - ref).abs() <= tol + least).all()), (r, s, slot[r], kv, float(((got - ref).abs() - tol).max()))
            assert bool(((gl - rl).abs() <= ltol).all()), (r, s, slot[r], kv, float((gl - rl).abs().max()))


def run_rows(w, counts, first=None, layer=None, q_type=BF16, out_type=BF16, most=60, slots=True, scale=1.5, least=0.0, **kw):
    layer = w.L - 1 if layer is None else layer
    start_d, slot_d, start, slot = w.rows(counts, first)
    n = len(slot)
    q = w.normal(n, w.Hq, D).mul(scale).to(q_type)
    out = torch.full((n + 2, w.Hq, D), 5.0, dtype=out_type, device=w.dev)
    lse = torch.full((n, w.Hq), math.nan, device=w.dev)
    w.md.attend_rows(layer, q, out[:n], start_d, row_slot=slot_d if slots else None, lse=lse, **kw)
    torch.cuda.synchronize()
    assert w.md.device_status() == 0
    assert (out[n:] == 5.0).all()
    some = None if n <= most else sorted({0, n - 1} | set(np.random.default_rng(n).choice(n, most, replace=False).tolist()))
    check_rows(w, layer, q, out[:n], lse, start, slot, some=some, least=least, **kw)
    return q, out[:n], lse, start_d, slot_d


TYPES = [(BF16, BF16), (torch.float32, torch.float32), (torch.float32, BF16), (BF16, torch.float32)]


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("types", TYPES, ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
def test_rows_of_prompts(types, coded, P):
    say("[rows]", types, coded, P)
    w = World(2, 12, 2, P, [300, 0, 1, 16, 65, 47], seed=51, coded=coded)
    run_rows(w, [300, 0, 1, 16, 65, 47], q_type=types[0], out_type=types[1], slots=False)
    run_rows(w, [20, 0, 1, 3, 64, 40], first=[133, 0, 0, 5, 0, 3], layer=0, q_type=types[0], out_type=types[1])


@pytest.mark.parametrize("shape", [(1, 1, 1), (3, 5, 5), (2, 16, 1), (1, 32, 8), (1, 14, 2)])
@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
def test_rows_head_layouts(types, shape):
    w = World(*shape, 16, [150, 0, 1, 290], seed=52)
    run_rows(w, [150, 0, 1, 290], q_type=types[0], out_type=types[1])


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("coded,aligned,quant", [(True, True, 0.0), (False, False, 0.6), (True, True, 0.6), (False, True, 0.0)])
def test_rows_holes_and_codes(coded, aligned, quant, P):
    say("[rows]", coded, aligned, quant, P)
    w = World(2, 12, 2, P, [300, 0, 1, 16, 800], seed=53, coded=coded, aligned=aligned, quant=quant)
    run_rows(w, [300, 0, 1, 16, 90])
    run_rows(w, [40, 0, 1, 16, 9], q_type=torch.float32, out_type=torch.float32, window=50, sinks=18)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 200), (16, 0), (17, 16), (64, 4), (129, 70), (5000, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_rows_windows(window, sinks, types):
    say("[rows window]", window, sinks, types)
    w = World(1, 4, 2, 16, [700, 3, 64, 0, 33], seed=54)
    run_rows(w, [400, 3, 64, 0, 20], q_type=types[0], out_type=types[1], window=window, sinks=sinks)
    run_rows(w, [3, 1, 2, 0, 5], first=[600, 0, 40, 0, 3], q_type=types[0], out_type=types[1], window=window, sinks=sinks)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1, 1], [5, 0], [7, 33]])
def test_few_rows_over_long_sessions(counts, types):
    """Work split over the slots and joined."""
    w = World(1, 12, 2, 64, [9000, 4100], seed=55)
    run_rows(w, counts, q_type=types[0], out_type=types[1])
    run_rows(w, counts, q_type=types[0], out_type=types[1], window=3000, sinks=5)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("counts", [[6, 2, 1, 0, 9], [11, 6, 0, 5, 80], [200, 60, 20, 0, 90]])
def test_parts_of_uneven_sessions(counts, types):
    """Long sessions are cut into more parts than short ones."""
    say("[parts]", counts, types)
    w = World(1, 12, 2, 16, [12000, 300, 40, 7, 2500], seed=59, coded=types[0] == BF16)
    run_rows(w, counts, q_type=types[0], out_type=types[1], most=40)
    run_rows(w, counts, q_type=types[0], out_type=types[1], window=900, sinks=20, most=40)


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("count", [5, 70])
def test_rows_of_any_slots(count, types):
    """Slots in no order, some twice: a tile's window covers more than its rows' number."""
    say("[any slots]", count, types)
    w = World(1, 8, 2, 16, [6000, 90], seed=60)
    start = np.array([0, count, count + 3])
    rng = np.random.default_rng(count)
    slot = np.concatenate([rng.integers(0, 6000, count), [89, 0, 0]])
    slot[1] = slot[0]
    for window, sinks in ((0, 0), (300, 17)):
        q = w.normal(count + 3, w.Hq, D).mul(1.5).to(types[0])
        out = torch.empty((count + 3, w.Hq, D), dtype=types[1], device=w.dev)
        lse = torch.empty((count + 3, w.Hq), device=w.dev)
        w.md.attend_rows(0, q, out, torch.as_tensor(start, dtype=torch.int32, device=w.dev),
                         row_slot=torch.as_tensor(slot, dtype=torch.int32, device=w.dev), lse=lse, window=window, sinks=sinks)
        torch.cuda.synchronize()
        assert w.md.device_status() == 0
        check_rows(w, 0, q, out, lse, start, slot, window=window, sinks=sinks)


def test_rows_of_many_sessions():
    lens = [(7 * i) % 40 for i in range(1024)]
    w = World(1, 2, 2, 16, lens, seed=56)
    run_rows(w, [min(n, 3) for n in lens])
    run_rows(w, lens, slots=False, most=200)


def test_longer_prompt():
    w = World(1, 8, 1, 16, [2500, 1300], seed=57, coded=False)
    run_rows(w, [2500, 1300], most=40)
    run_rows(w, [2500, 1300], most=40, window=777, sinks=33)


def test_growing_logits():
    """Maxima that grow along a row by little and by much: the running one is
    followed late, the results stay."""
    for grow in (0.002, 0.05, 0.5):
        w = World(1, 2, 1, 16, [600], seed=58, coded=False)
        ramp = torch.arange(600, dtype=torch.float64)[:, None, None, None] * grow
        w.k[0] = (w.k[0] * 0.05 + ramp / math.sqrt(D)).float().to(BF16).double()
        ids = torch.as_tensor(w.ids[0], device=w.dev)
        full = torch.zeros((len(ids) * 16, 1, 1, D), dtype=BF16, device=w.dev)
        full[:600] = w.k[0].to(BF16).to(w.dev)
        w.cache.k_pool[ids] = PagedCache.to_pool_layout(full.view(-1, 16, 1, 1, D))
        for types in TYPES[:2]:
            start_d, slot_d, start, slot = w.rows([600])
            q = torch.ones((600, 2, D), device=w.dev).to(types[0])
            q[:, 1] *= -1
            out, lse = torch.empty_like(q).to(types[1]), torch.empty((600, 2), device=w.dev)
            w.md.attend_rows(0, q, out, start_d, lse=lse)
            check_rows(w, 0, q, out, lse, start, slot, some=list(range(0, 600, 23)))


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("many", [True, False])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(many, coded, types):
    """Rows before such a value, and rows whose window is past it, keep their results."""
    w = World(1, 2, 1, 16, [200], seed=59, coded=coded, quant=0.5)
    ids = w.ids[0]
    bad = [150] if coded else [33, 150]
    for t in bad:
        page, x = int(ids[t // 16]), (math.inf if t == 33 else math.nan)
        if coded:
            w.cache.v_scale[page] = math.nan
            w.v[0][t // 16 * 16:t // 16 * 16 + 16] = math.nan
        else:
            y = PagedCache.from_value_layout(w.cache.v_pool[page:page + 1]).contiguous()
            y[0, t % 16] = x
            w.cache.v_pool[page:page + 1] = PagedCache.to_value_layout(y)
            w.v[0][t] = x
    counts, first = ([200], None) if many else ([2], [141])
    start_d, slot_d, start, slot = w.rows(counts, first)
    q = w.normal(len(slot), 2, D).to(types[0])
    for kw in (dict(), dict(window=20, sinks=2)):
        out, lse = torch.zeros((len(slot), 2, D), dtype=types[1], device=w.dev), torch.zeros((len(slot), 2), device=w.dev)
        w.md.attend_rows(0, q, out, start_d, row_slot=slot_d, lse=lse, **kw)
        sees_bad = [bool((visible(w.live[0], t, kw.get("window", 0), kw.get("sinks", 0)).double()[:, None, None]
                          * torch.where(w.v[0][:, 0].isfinite(), 0.0, 1.0)).any()) for t in slot]
        check_rows(w, 0, q, out, lse, start, slot, some=[r for r in range(len(slot)) if not sees_bad[r]], **kw)
        for r in range(len(slot)):
            assert bool(out[r].isfinite().all()) != sees_bad[r], (r, slot[r])


@pytest.mark.parametrize("types", TYPES[:2], ids=["bf16", "f32"])
@pytest.mark.parametrize("power", [-122, -60, 60, 110])
@pytest.mark.parametrize("some", [True, False])
def test_scales_of_any_size(some, power, types):
    """Scales of 8-bit values that are far from 1, of all blocks or of one."""
    say("[scales]", some, power, types)
    w = World(1, 4, 2, 16, [330, 40], seed=61)
    for s in range(2):
        blocks = [1] if some else range(len(w.ids[s]))
        for b in blocks:
            scale = w.cache.v_scale[int(w.ids[s][b])]   # [L][Hkv][1]
            before = scale.cpu().double()
            scale *= 2.0 ** power
            w.v[s][16 * b:16 * b + 16] *= scale.cpu().double() / before   # (a small one loses bits)
    # (results below 2^-126 are multiples of 2^-133 in bf16: off by at most half of it)
    run_rows(w, [330, 40], q_type=types[0], out_type=types[1], least=2.0 ** -134)
    run_rows(w, [3, 2], q_type=types[0], out_type=types[1], window=30, sinks=20, least=2.0 ** -134)


def test_keys_that_are_not_finite_and_nan_queries_stay_where_they_are_seen():
    w = World(1, 2, 1, 16, [100], seed=60, coded=False)
    page = int(w.ids[0][4])
    y = PagedCache.from_pool_layout(w.cache.k_pool[page:page + 1]).contiguous()
    y[0, 6] = math.nan
    w.cache.k_pool[page:page + 1] = PagedCache.to_pool_layout(y)
    w.k[0][70] = math.nan
    start_d, slot_d, start, slot = w.rows([100])
    for types in TYPES[:2]:
        q = w.normal(100, 2, D).to(types[0])
        q[20, 1, 5] = math.nan
        out, lse = torch.zeros((100, 2, D), dtype=types[1], device=w.dev), torch.zeros((100, 2), device=w.dev)
        w.md.attend_rows(0, q, out, start_d, lse=lse)
        assert out[20, 1].isnan().all() and lse[20, 1].isnan() and out[20, 0].isfinite().all()
        assert out[70:].isnan().all()
        rows = [r for r in range(70) if r != 20]
        check_rows(w, 0, q, out, lse, start, slot, some=rows)


def test_rows_that_see_nothing():
    w = World(1, 2, 1, 16, [40, 5], seed=61)
    q = w.normal(8, 2, D)
    for types in TYPES[:2]:
        out, lse = torch.full((8, 2, D), 5.0, dtype=types[1], device=w.dev), torch.full((8, 2), 5.0, device=w.dev)
        w.md.attend_rows(0, q.to(types[0]), out, w.i32([1, 4, 6]), row_slot=w.i32([0, 0, -1, 40, 5, 4, 0, 0]), lse=lse)
        assert w.md.device_status() == B.MD_DEV_BAD_ROW
        none = [bool((out[i] == 0).all() and (lse[i] == -math.inf).all()) for i in range(8)]
        left = [bool((out[i] == 5).all() and (lse[i] == 5).all()) for i in range(8)]
        assert none == [False, False, True, True, True, False, False, False] and left == [True] + [False] * 5 + [True, True]


def test_inconsistent_sessions_are_left_out():
    w = World(1, 2, 1, 16, [40, 40, 40], seed=62)
    w.cache.n_tokens[0] = 4000
    w.cache.page_table[1, 1] = w.cache.n_phys
    q = w.normal(60, 2, D).to(BF16)
    k, v = (w.normal(60, 1, D, dtype=BF16) for _ in range(2))
    start, out = w.i32([0, 20, 40, 60]), torch.full((60, 2, D), 5.0, dtype=BF16, device=w.dev)
    before = w.cache.k_pool.clone()
    w.md.write_rows(0, w.i32([0, 20, 20, 20]), k[:20], v[:20])
    assert w.md.device_status() == B.MD_DEV_CORRUPT
    assert torch.equal(before.view(torch.uint8), w.cache.k_pool.view(torch.uint8))
    w.md.attend_rows(0, q, out, start)
    assert w.md.device_status() & B.MD_DEV_CORRUPT
    assert (out[:20] == 0).all() and out[20:].isfinite().all() and (out[40:] != 5).any()
    w.md.read_rows(0, start, k, v)
    assert w.md.device_status() & B.MD_DEV_CORRUPT
    assert (k[:20] == 0).all()


def test_the_same_bits_every_time():
    w = World(1, 12, 2, 16, [3000, 1, 500], seed=63)
    for counts in ([4, 1, 3], [700, 1, 300]):
        first = None
        start_d, slot_d, start, slot = w.rows(counts)
        q = w.normal(len(slot), 12, D)
        for types in TYPES[:2]:
            ref = None
            for _ in range(4):
                out, lse = torch.empty_like(q).to(types[1]), torch.empty(q.shape[:2], device=w.dev)
                w.md.attend_rows(0, q.to(types[0]), out, start_d, lse=lse)
                if ref is None:
                    ref = out, lse
                assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


def test_strided_rows_and_untouched_neighbours():
    w = World(2, 4, 2, 16, [200, 30], seed=64)
    start_d, slot_d, start, slot = w.rows([50, 30])
    for types in TYPES[:2]:
        q = torch.full((80, 3, 4, D), math.nan, device=w.dev).to(types[0])
        q[:, 1] = w.normal(80, 4, D).to(types[0])
        out = torch.full((80, 3, 4, D), 5.0, device=w.dev).to(types[1])
        lse = torch.zeros((80, 4), device=w.dev)
        w.md.attend_rows(1, q[:, 1], out[:, 1], start_d, lse=lse)
        check_rows(w, 1, q[:, 1], out[:, 1], lse, start, slot, some=range(0, 80, 7))
        assert (out[:, 0] == 5).all() and (out[:, 2] == 5).all()
        plain = torch.empty((80, 4 * D), device=w.dev).to(types[1])
        w.md.attend_rows(1, q[:, 1].reshape(80, -1), plain, start_d)
        assert torch.equal(plain.view(80, 4, D), out[:, 1])


# ---- The same where there are many columns (more than 2,048, and more than 128
# a session): bf16 rows then take the kernel of 256 columns a workgroup.

@pytest.mark.parametrize("coded", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 200), (16, 0), (17, 16), (64, 4), (129, 70), (5000, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_many_columns_windows(window, sinks, coded):
    say("[columns window]", window, sinks, coded)
    w = World(1, 16, 1, 16, [700, 3, 64, 0, 33], seed=81, coded=coded)
    run_rows(w, [400, 3, 64, 0, 20], window=window, sinks=sinks)


@pytest.mark.parametrize("shape", [(1, 16, 1), (2, 32, 2), (1, 14, 2), (1, 32, 8)])
def test_many_columns_head_layouts(shape):
    w = World(*shape, 64, [520, 0, 1, 290], seed=82, quant=0.5)
    run_rows(w, [520, 0, 1, 290])


@pytest.mark.parametrize("power", [-122, -60, 60, 110])
@pytest.mark.parametrize("some", [True, False])
def test_many_columns_scales(some, power):
    say("[columns scales]", some, power)
    w = World(1, 16, 1, 16, [330, 40], seed=83)
    for s in range(2):
        for b in [1] if some else range(len(w.ids[s])):
            scale = w.cache.v_scale[int(w.ids[s][b])]
            before = scale.cpu().double()
            scale *= 2.0 ** power
            w.v[s][16 * b:16 * b + 16] *= scale.cpu().double() / before
    run_rows(w, [330, 40], least=2.0 ** -134)


@pytest.mark.parametrize("coded", [True, False])
def test_many_columns_values_that_are_not_finite(coded):
    w = World(1, 16, 1, 16, [200], seed=84, coded=coded, quant=0.5)
    for t in [150] if coded else [33, 150]:
        page = int(w.ids[0][t // 16])
        if coded:
            w.cache.v_scale[page] = math.nan
            w.v[0][t // 16 * 16:t // 16 * 16 + 16] = math.nan
        else:
            y = PagedCache.from_value_layout(w.cache.v_pool[page:page + 1]).contiguous()
            y[0, t % 16] = w.v[0][t] = math.inf if t == 33 else math.nan
            w.cache.v_pool[page:page + 1] = PagedCache.to_value_layout(y)
    start_d, slot_d, start, slot = w.rows([200])
    q = w.normal(200, 16, D).to(BF16)
    for kw in (dict(), dict(window=20, sinks=2)):
        out, lse = torch.zeros((200, 16, D), dtype=BF16, device=w.dev), torch.zeros((200, 16), device=w.dev)
        w.md.attend_rows(0, q, out, start_d, lse=lse, **kw)
        bad = ~w.v[0][:, 0, 0].isfinite().all(1)
        sees_bad = [bool((visible(w.live[0], t, kw.get("window", 0), kw.get("sinks", 0)) & bad).any()) for t in slot]
        check_rows(w, 0, q, out, lse, start, slot, some=[r for r in range(200) if not sees_bad[r]][::3], **kw)
        for r in range(200):
            assert bool(out[r].isfinite().all()) != sees_bad[r], (r, slot[r])


def test_many_columns_keys_that_are_not_finite():
    w = World(1, 16, 1, 16, [200], seed=85, coded=False)
    page = int(w.ids[0][4])
    y = PagedCache.from_pool_layout(w.cache.k_pool[page:page + 1]).contiguous()
    y[0, 6] = math.nan
    w.cache.k_pool[page:page + 1] = PagedCache.to_pool_layout(y)
    w.k[0][70] = math.nan
    start_d, slot_d, start, slot = w.rows([200])
    q = w.normal(200, 16, D).to(BF16)
    q[20, 1, 5] = math.nan
    out, lse = torch.zeros((200, 16, D), dtype=BF16, device=w.dev), torch.zeros((200, 16), device=w.dev)
    w.md.attend_rows(0, q, out, start_d, lse=lse)
    assert out[20, 1].isnan().all() and lse[20, 1].isnan() and out[20, 0].isfinite().all()
    assert out[70:].isnan().all()
    check_rows(w, 0, q, out, lse, start, slot, some=[r for r in range(70) if r != 20])


@pytest.mark.parametrize("grow", [0.002, 0.05, 0.5])
def test_many_columns_growing_logits(grow):
    w = World(1, 16, 1, 16, [600], seed=86, coded=False)
    ramp = torch.arange(600, dtype=torch.float64)[:, None, None, None] * grow
    w.k[0] = (w.k[0] * 0.05 + ramp / math.sqrt(D)).float().to(BF16).double()
    ids = torch.as_tensor(w.ids[0], device=w.dev)
    full = torch.zeros((len(ids) * 16, 1, 1, D), dtype=BF16, device=w.dev)
    full[:600] = w.k[0].to(BF16).to(w.dev)
    w.cache.k_pool[ids] = PagedCache.to_pool_layout(full.view(-1, 16, 1, 1, D))
    start_d, slot_d, start, slot = w.rows([600])
    q = torch.ones((600, 16, D), dtype=BF16, device=w.dev)
    q[:, 1::2] *= -1
    out, lse = torch.empty_like(q), torch.empty((600, 16), device=w.dev)
    w.md.attend_rows(0, q, out, start_d, lse=lse)
    check_rows(w, 0, q, out, lse, start, slot, some=list(range(0, 600, 23)))


def test_many_columns_rows_that_do_not_count():
    """Rows of nobody, of slots that are not there, of sessions that make no sense."""
    w = World(1, 16, 1, 16, [300, 5, 40, 40], seed=87)
    w.cache.n_tokens[2] = 4000
    n = 260
    start = w.i32([1, 200, 203, 223, 243])
    slot = np.concatenate([[0], np.arange(100, 299), [-1, 5, 4], np.arange(20), np.arange(20), np.zeros(17, np.int64)])
    q = w.normal(n, 16, D).to(BF16)
    out, lse = torch.full((n, 16, D), 5.0, dtype=BF16, device=w.dev), torch.full((n, 16), 5.0, device=w.dev)
    w.md.attend_rows(0, q, out, start, row_slot=w.i32(slot.tolist()), lse=lse)
    assert w.md.device_status() == B.MD_DEV_BAD_ROW | B.MD_DEV_CORRUPT
    none = [i for i in range(n) if bool((out[i] == 0).all() and (lse[i] == -math.inf).all())]
    left = [i for i in range(n) if bool((out[i] == 5).all() and (lse[i] == 5).all())]
    assert none == [200, 201] + list(range(203, 223)) and left == [0] + list(range(243, 260))
    rows = list(range(1, 200, 9)) + [202] + list(range(223, 243, 5))
    check_rows(w, 0, q[1:243], out[1:243], lse[1:243], np.array([0, 199, 202, 222, 242]), slot[1:243], some=[r - 1 for r in rows])


def test_many_columns_strided_rows():
    w = World(2, 32, 2, 16, [200, 30], seed=88)
    start_d, slot_d, start, slot = w.rows([140, 30])
    q = torch.full((170, 3, 32, D), math.nan, dtype=BF16, device=w.dev)
    q[:, 1] = w.normal(170, 32, D).to(BF16)
    out = torch.full((170, 3, 32, D), 5.0, dtype=BF16, device=w.dev)
    lse = torch.zeros((170, 32), device=w.dev)
    w.md.attend_rows(1, q[:, 1], out[:, 1], start_d, lse=lse)
    check_rows(w, 1, q[:, 1], out[:, 1], lse, start, slot, some=range(0, 170, 11))
    assert (out[:, 0] == 5).all() and (out[:, 2] == 5).all()


def test_many_columns_replayed_between_few():
    """One work space for both kernels and their parts, captured and replayed."""
    side = torch.cuda.Stream()
    w = World(1, 16, 1, 16, [3000, 1100], seed=89, stream=side)
    many, few = w.rows([200, 100]), w.rows([5, 2])
    qs = [w.normal(n, 16, D).to(BF16) for n in (300, 7)]
    outs = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()

    def calls():
        w.md.attend_rows(0, qs[0], outs[0], many[0], row_slot=many[1])
        w.md.attend_rows(0, qs[1], outs[1], few[0], row_slot=few[1], window=1500, sinks=3)

    calls()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    lse = torch.zeros((300, 16), device=w.dev)
    w.md.attend_rows(0, qs[0], outs[0], many[0], row_slot=many[1], lse=lse)
    torch.cuda.synchronize()
    check_rows(w, 0, qs[0], outs[0], lse, many[2], many[3], some=range(0, 300, 29))


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("coded", [True, False])
def test_pools_past_32_bits(coded):
    """Pages whose keys and values lie more than 2^32 elements into the pools."""
    say("[large pools]", coded)
    w = World(1, 32, 2, 16, [300, 40], seed=91, coded=coded, fill=False, spare=800000)
    assert max(int(i) for ids in w.ids for i in ids) * 2 * 16 * D > 2 ** 32
    start_d, slot_d, start, slot = w.rows([300, 40])
    k, v = kv_rows(w, start, slot, 0)
    w.md.write_rows(0, start_d, k, v, row_slot=slot_d)
    back = [torch.zeros((340, 2, D), device=w.dev) for _ in "kv"]
    w.md.read_rows(0, start_d, *back, row_slot=slot_d)
    torch.cuda.synchronize()
    session = np.repeat([0, 1], [300, 40])
    assert torch.equal(back[0], k.float())
    want = torch.stack([w.v[s][t, 0] for s, t in zip(session, slot)])
    assert torch.equal(back[1].cpu(), want.float())   # (codes: the product of scale and code, rounded once)
    run_rows(w, [300, 40], most=20)
    run_rows(w, [4, 3], window=100, sinks=20)
    q, out = w.normal(2, 32, D), torch.zeros((2, 32, D), device=w.dev)
    w.md.attend(0, q, out)
    rows = torch.zeros((2, 32, D), device=w.dev)
    w.md.attend_rows(0, q, rows, w.i32([0, 1, 2]))
    torch.cuda.synchronize()
    assert w.md.device_status() == 0
    assert float((out - rows).abs().max()) < 1e-4


def test_two_handles_and_another_stream():
    """Calls on a handle's own stream, whatever stream is current."""
    side = torch.cuda.Stream()
    w = World(1, 4, 2, 16, [600, 40], seed=71)
    other = MemDecay(w.cache, torch.ones((2, 7)), torch.ones((2, 7)), rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0, stream=side)
    start_d, slot_d, start, slot = w.rows([9, 4])
    q = w.normal(13, 4, D)
    outs = [torch.zeros((13, 4, D), device=w.dev) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        w.md.attend_rows(0, q, outs[0], start_d)
        other.attend_rows(0, q, outs[1], start_d)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    assert w.md._rows_ws.data_ptr() != other._rows_ws.data_ptr()


def test_captured_calls_replay():
    w = World(2, 4, 2, 16, [700, 33], seed=72)
    start_d, slot_d, start, slot = w.rows([28, 1])   # whole blocks, so that writing them again changes nothing else
    n = 29
    side = torch.cuda.Stream()
    md = MemDecay(w.cache, torch.ones((2, 7)), torch.ones((2, 7)), rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0, stream=side)
    k, v = (w.normal(n, 2, D, dtype=BF16) for _ in range(2))
    q, out, lse = w.normal(n, 4, D).to(BF16), torch.zeros((n, 4, D), dtype=BF16, device=w.dev), torch.zeros((n, 4), device=w.dev)
    tq, tout = w.normal(2, 4, D), torch.zeros((2, 4, D), device=w.dev)
    back = torch.zeros((n, 2, D), device=w.dev)

    def calls():
        md.write_rows(1, start_d, k, v, row_slot=slot_d)
        md.attend_rows(1, q, out, start_d, row_slot=slot_d, lse=lse, window=300, sinks=2)
        md.attend(1, tq, tout, window=100, sinks=1)
        md.read_rows(1, start_d, v_out=back, row_slot=slot_d)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            md.attend_rows(1, q, out, start_d)
    torch.cuda.synchronize()
    calls()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls()
    for i in range(4):
        k.copy_(w.normal(n, 2, D, dtype=BF16))
        v.copy_(w.normal(n, 2, D, dtype=BF16))
        q.copy_(w.normal(n, 4, D).to(BF16))
        tq.copy_(w.normal(2, 4, D))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, tout, back)]
        for x in (out, lse, tout, back):
            x.zero_()
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, tout, back))), i
        torch.ones(1000, device=w.dev).sum().item()


@pytest.mark.parametrize("kw", [dict(), dict(P=64), dict(aligned=True), dict(quant=True), dict(coded=False)],
                         ids=["p16", "p64", "aligned", "quant", "bf16"])
def test_prompts_in_chunks_then_steps(kw):
    """Prompts enter in chunks, layer by layer (heads, rows written, attention),
    then steps append tokens and evict pages: every result against 64 bits, on
    what the cache then holds."""
    P, aligned, quant, coded = kw.get("P", 16), kw.get("aligned", False), kw.get("quant", False), kw.get("coded", True)
    L, Hq, Hkv = 2, 4, 2
    w = World(L, Hq, Hkv, P, [100, 37, 64], seed=73, coded=coded, aligned=aligned, fill=False, spare=10, extra=10,
              quant_threshold=math.inf if quant else 0.0)
    c, md = w.cache, w.md
    inv = torch.as_tensor(10000.0 ** (-np.arange(0, D, 2) / D), device=w.dev)
    wq, wk = (torch.rand(D, generator=w.g).to(w.dev) + 0.5 for _ in range(2))
    lens = np.array([100, 37, 64])
    for lo, hi in ((0, 30), (30, 64), (64, 100)):
        n = np.clip(lens, lo, hi) - lo
        first = [int(np.flatnonzero(w.live[s])[lo]) if n[s] else w.slots[s] for s in range(3)]
        start_d, slot_d, start, slot = w.rows(n, first)
        session = np.repeat(np.arange(3), n)
        token = np.concatenate([np.arange(lo, lo + x) for x in n])
        for layer in range(L):
            qkv = w.normal(len(slot), (Hq + 2 * Hkv) * D).to(BF16)
            q = torch.empty((len(slot), Hq, D), device=w.dev)
            k, v = (torch.empty((len(slot), Hkv, D), dtype=BF16, device=w.dev) for _ in range(2))
            md.norm_rope(qkv, q, k, v, q_weight=wq, k_weight=wk, inv_freq=inv, position=w.i32(token))
            md.write_rows(layer, start_d, k, v, row_slot=slot_d)
            for r, (s, t) in enumerate(zip(session, slot)):
                w.k[s][t, layer] = k[r].double().cpu()
                w.v16[s][t, layer] = v[r].float().cpu()
            for s in range(3):
                upto = int(slot[session == s].max()) + 1 if (session == s).any() else 0
                if upto:
                    x = w.v16[s][:upto, layer]
                    w.v[s][:upto, layer] = quantise_slots(x) if coded else x.double()
            out, lse = torch.empty((len(slot), Hq, D), dtype=BF16, device=w.dev), torch.empty((len(slot), Hq), device=w.dev)
            qb = q.to(BF16)
            md.attend_rows(layer, qb, out, start_d, row_slot=slot_d, lse=lse, window=50 if layer else 0, sinks=3)
            check_rows(w, layer, qb, out, lse, start, slot, window=50 if layer else 0, sinks=3, some=range(0, len(slot), 5))
    assert md.device_status() == 0
    c.budget.fill_(60)
    for step in range(25):
        nk, nv = (w.normal(3, L, Hkv, D, dtype=BF16) for _ in range(2))
        q = w.normal(3, 1, L, Hq, D)
        refs = []
        for s in range(3):   # what the cache holds now, read back
            n = int(c.n_tokens[s])
            slots = w.i32(np.arange(n))
            start = np.zeros(4, int)
            start[s + 1:] = n
            kr, vr = (torch.empty((n, Hkv, D), device=w.dev) for _ in range(2))
            per = []
            for layer in range(L):
                md.read_rows(layer, w.i32(start), kr, vr, row_slot=slots)
                per.append((kr.double().cpu(), vr.double().cpu()))
            page = c.page_table[s, :int(c.n_pages[s])].long()
            live = (c.region[page].flatten()[:n] != B.MD_REGION_HOLE).cpu().numpy()
            refs.append((per, live))
        for layer in range(L):
            kw2 = dict(window=40, sinks=2) if layer else {}
            out, lse = torch.empty((3, Hq, D), device=w.dev), torch.empty((3, Hq), device=w.dev)
            md.attend(layer, q[:, 0, layer], out, new_k=nk[:, layer].contiguous(), new_v=nv[:, layer].contiguous(), lse=lse, **kw2)
            w.k = [torch.stack([p[0] for p in per], 1) for per, _ in refs]
            w.v = [torch.stack([p[1] for p in per], 1) for per, _ in refs]
            w.live = [live for _, live in refs]
            check_token(w, layer, q[:, 0, layer], out, lse, nk[:, layer], nv[:, layer], **kw2)
        md.observe(step, q, nk, torch.as_tensor(w.rng.integers(1, 7, 3).astype(np.uint8), device=w.dev))
        md.append_values(nv)
        md.score()
        md.select_compact()
        assert md.device_status() & ~B.MD_W_BUDGET_INFEASIBLE == 0
    if quant:
        assert int(c.page_format.sum()) > 0


# ---------------------------------------------------------------- refusals

def test_refusals():
    w = World(1, 4, 2, 16, [40, 5], seed=81)
    md = w.md
    k = torch.zeros((6, 2, D), dtype=BF16, device=w.dev)
    start, slot = w.i32([0, 3, 6]), w.i32([0, 1, 2, 0, 1, 2])
    q, out = torch.zeros((6, 4, D), device=w.dev), torch.zeros((6, 4, D), device=w.dev)

    def refused(fn, *a, **kw):
        with pytest.raises((ValueError, B.MemDecayError)):
            fn(*a, **kw)

    refused(md.write_rows, 0, start)
    refused(md.write_rows, 0, start, k.float(), k)
    refused(md.write_rows, 0, start, k, k[:5])
    refused(md.write_rows, 0, start[:2], k, k)
    refused(md.write_rows, 0, start.long(), k, k)
    refused(md.write_rows, 0, start, k, k, row_slot=slot[:5])
    refused(md.write_rows, 1, start, k, k)
    refused(md.write_rows, -1, start, k, k)
    refused(md.write_rows, 0, start, k, k.transpose(1, 2).contiguous().transpose(1, 2))
    refused(md.write_rows, 0, start, k.cpu(), k.cpu())
    refused(md.read_rows, 0, start, k.half(), k.half())
    refused(md.read_rows, 0, start, k, k.float())
    refused(md.read_rows, 0, start)
    refused(md.attend_rows, 0, q.half(), out, start)
    refused(md.attend_rows, 0, q, out[:5], start)
    refused(md.attend_rows, 0, q, out, start, window=-1)
    refused(md.attend_rows, 0, q, out, start, window=1, sinks=-1)
    refused(md.attend_rows, 3, q, out, start)
    refused(md.attend_rows, 0, q, out, start, lse=torch.zeros(5, device=w.dev))
    t, b, n = torch.zeros((2, 4, D), device=w.dev), w.i32(np.zeros((2, 2, 1))), w.i32(np.zeros((2, 2)))
    refused(md.attend, 0, t, t.clone(), window=-1)
    refused(md.attend, 0, t, t.clone(), window=4, blocks=b, block_count=n)
    md.write_rows(0, w.i32([0, 0, 0]), k[:0], k[:0])
    md.read_rows(0, w.i32([0, 0, 0]), k[:0], k[:0])
    md.attend_rows(0, q[:0], out[:0], w.i32([0, 0, 0]))
    assert md.device_status() == 0
    bare = PagedCache(L=1, Hq=4, Hkv=2, d=D, P=16, S=2, max_pages=4, n_phys=8)
    ones = torch.ones((2, 7))
    none = MemDecay(bare, ones, ones, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0)
    refused(none.attend_rows, 0, q, out, start)
    refused(none.read_rows, 0, start, k, k)
    refused(none.write_rows, 0, start, k, k)
    none.write_rows(0, start, k)   # keys need no values
    assert none.device_status() == B.MD_DEV_BAD_ROW


def test_offload_handles_refuse_rows():
    c = PagedCache(L=1, Hq=4, Hkv=2, d=D, P=16, S=1, max_pages=4, n_phys=8, offload_pages=2, values="e4m3")
    ones = torch.ones((1, 7))
    md = MemDecay(c, ones, ones, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=0)
    k = torch.zeros((1, 2, D), dtype=BF16, device=c.device)
    start = torch.tensor([0, 1], dtype=torch.int32, device=c.device)
    q = torch.zeros((1, 4, D), device=c.device)
    for call in (lambda: md.write_rows(0, start, k, k), lambda: md.read_rows(0, start, k, k),
                 lambda: md.attend_rows(0, q, q.clone(), start), lambda: md.attend(0, q, q.clone()),
                 lambda: md.append_values(k[:, None].contiguous())):
        with pytest.raises(B.MemDecayError) as e:
            call()
        assert e.value.status == B.MD_E_UNSUPPORTED
