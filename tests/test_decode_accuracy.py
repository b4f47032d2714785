"""How near the attention over the paged cache comes to its definition, in
bounds tight enough that a lost or doubled token, a weight of fewer bits or a
query of fewer bits does not fit in them.  That they are is shown first, on
the CPU, with each mistake planted in the 64-bit oracle.

Three kinds of input, tolerances derived before any run (u = 2^-24, half a
float32 step, relative):

* counted: a query of zeros makes every weight exactly 1, and values are whole
  numbers from 1 to 3 of either sign, so that sums of up to 2^24 / 3 tokens
  are exact in any order.  Left are the reciprocal of the number of tokens
  and the product with it: 2 u.  One token more or less changes a sum by at
  least 1 of at most 3 n: far more up to n = 2^20.  The log-sum is
  log2(n) ln 2: a logarithm of two units, the product and its constant, 6 u
  of it at most; n - 1 instead of n moves it by 1 / n.
* two tokens: query (a, 0, ..), keys (1, 0, ..) and zero, values 1 and -1.  The
  logit a is exact (the three bf16 terms of a add up to it), its product with
  the scale, |y| <= 4 in base 2, takes a rounding and the constant's: |y| 2 u
  ln 2 <= 5.6 u of the weight p, its exponential 2 u, its three bf16 terms
  u / 4.  out = (1 - p) / (1 + p) moves by at most half of that, 4 u; the sum of
  the weights, the reciprocal and the last product take u each, the sum of the
  values, to which the terms are added one after another, 3 u: 10 u in all.
  (Tokens that do not lie in one tile of 16 have their weights from the float32
  factors that join two results, and no terms.)  The log-sum: 5.6 u from y and
  the exponential's and sum's 3 u (in l), 6 u of itself.
* drawn: a logit is 384 exact products added in float32; each rounding is at
  most u of the partial sum so far, whose mean square is half of the square
  sum |p|^2 of all, and roundings are uniform and of either sign:
  u |p| sqrt(384 / 2 / 3) = 8 u |p|, six times which is taken, d = 48 u |p| /
  sqrt(128) for the token with the largest |p|.  An output moves by at most
  sum_i w_i d (|v_i| + |out|); exponentials and sums take 2^-20 of sum_i w_i |v_i|.
"""
import math

import numpy as np
import pytest
import torch

import decode_oracle as O
from paper_2607_10582_amd.cache import PagedCache
from test_gpu_decode import BF16, D, LENS, World, say

U = 2.0 ** -24


# ------------------------------------------------------------------ the bounds

def counted_bounds(v):
    """Values [n][d] of the tokens that count -> (out, its bound, lse, its bound)."""
    n = v.shape[0]
    out = v.double().sum(0) / n
    return out, 2 * U * out.abs(), math.log(n), 6 * U * math.log(n)


def pair_bounds():
    return 10 * U, lambda lse: 9 * U + 6 * U * abs(lse)


def drawn_bounds(q, k, v):
    """One head group -> (out, its bound, lse, its bound)."""
    q, k, v = q.double(), k.double(), v.double()
    out, lse = O.attend(q, k, v)
    w = torch.exp(q @ k.T / math.sqrt(D) - lse[:, None])
    d = 48 * U * ((q * q) @ (k * k).T).sqrt().amax(1, keepdim=True) / math.sqrt(D)
    a = w @ v.abs()
    return out, d * (a + out.abs()) + 2.0 ** -20 * a, lse, (d[:, 0] + 2.0 ** -20 * (1 + lse.abs()))


def terms(x, n, cut):
    """x as the sum of its first n bf16 terms, each cut off (a query's) or
    rounded (a weight's)."""
    x = x.float()
    total = torch.zeros_like(x, dtype=torch.float64)
    for _ in range(n):
        t = (x.view(torch.int32) & -65536).view(torch.float32) if cut else x.to(BF16).float()
        total += t.double()
        x = x - t
    return total


def planted(q, k, v, query=3, weight=3, lost=(), twice=()):
    """The attention of one head group with a mistake in it."""
    q, k, v = terms(q, query, True), k.double(), v.double()
    count = torch.ones(k.shape[0], dtype=torch.float64)
    count[list(lost)] = 0
    count[list(twice)] = 2
    x = q @ k.T / math.sqrt(D)
    p = torch.exp(x - x.max(1, keepdim=True).values) * count
    total = p.sum(1, keepdim=True)
    return (terms(p, weight, False) if weight < 3 else p) @ v / total, x.max(1).values + torch.log(total[:, 0])


def whole(n, gen, *shape):
    """Whole numbers from 1 to 3 of either sign."""
    return (torch.randint(1, 4, (n, *shape), generator=gen) * (1 - 2 * torch.randint(0, 2, (n, *shape), generator=gen))).float()


# ------------------------------------------------------------------ that they are tight

@pytest.mark.parametrize("n", [2, 17, 450, 5000, 131068])
def test_counted_bounds_tell_every_token(n):
    g = torch.Generator().manual_seed(n)
    v = whole(n, g, D)
    out, tol, lse, ltol = counted_bounds(v)
    rng = np.random.default_rng(n)
    for t in [0, n - 1, *rng.integers(0, n, 6)]:
        for m, s in ((n - 1, v.double().sum(0) - v[t]), (n + 1, v.double().sum(0) + v[t])):
            assert bool(((s / m - out).abs() > tol).any()) and abs(math.log(m) - lse) > ltol
        # lost, and another one twice
        s = v.double().sum(0) - v[t] + v[(t + 1) % n]
        assert bool(((s / n - out).abs() > tol).any())


def pair_inputs(gen, S, Hq):
    """a: logits of up to 4 in base 2, with all their 24 bits."""
    a = (torch.rand((S, Hq), generator=gen) * 2 - 1) * (4.0 * math.log(2) * math.sqrt(D))
    return a * (1 - 2.0 ** -20)


def pair_exact(a, **kw):
    k, v = torch.zeros((2, D)), torch.ones((2, 1))
    k[0, 0], v[1] = 1, -1
    q = torch.zeros((a.numel(), D))
    q[:, 0] = a.flatten()
    return planted(q, k, v, **kw) if kw else O.attend(q, k, v)


def test_pair_bounds_tell_the_bits_of_weights_and_queries():
    a = pair_inputs(torch.Generator().manual_seed(1), 64, 4)
    tol, ltol = pair_bounds()
    ref, lse = pair_exact(a)
    same, l3 = pair_exact(a, query=3)
    assert float((same - ref).abs().max()) < 1e-12 and float((l3 - lse).abs().max()) < 1e-12
    for kw in (dict(weight=1), dict(weight=2), dict(query=1), dict(query=2)):
        off, loff = pair_exact(a, **kw)
        assert float((off - ref).abs().max()) > 1.5 * tol, kw
        if "query" in kw:
            assert bool(((loff - lse).abs() > 2 * torch.tensor([ltol(float(x)) for x in lse])).any()), kw


@pytest.mark.parametrize("n", [450, 5000, 20011])
def test_drawn_bounds_tell_steps_and_single_terms(n):
    g = torch.Generator().manual_seed(n)
    q, k, v = torch.randn((6, D), generator=g) * 2, torch.randn((n, D), generator=g).to(BF16), torch.randn((n, D), generator=g).to(BF16)
    out, tol, lse, ltol = drawn_bounds(q, k, v)
    rng = np.random.default_rng(n)
    steps = [range(32 * i, min(n, 32 * i + 32)) for i in [0, (n - 1) // 32, *rng.integers(0, n // 32, 4)]]
    for kw in [dict(weight=1), dict(query=1)] + [dict(lost=s) for s in steps] + [dict(twice=s) for s in steps]:
        off, _ = planted(q, k, v, **kw)
        assert bool(((off - out).abs() > tol).any()), kw


# ------------------------------------------------------------------ on the device

def set_values(w, make):
    """Other values for a world's tokens, NaN in the slots without one."""
    c = w.cache
    for s in range(w.S):
        n = w.v[s].shape[0]
        if n == 0:
            continue
        w.v[s] = make(n, w.g, w.L, w.Hkv, D)
        region = w.regions[s] if w.aligned else None
        c.load_values(s, w.v[s].to(BF16), region)
        pos = PagedCache.positions(w.regions[s], w.P, w.aligned)
        dead = torch.as_tensor(np.setdiff1d(np.arange(w.pages[s] * w.P), pos), device=w.dev)
        own = c.page_table[s, :w.pages[s]].long()
        x = PagedCache.from_value_layout(c.v_pool[own])
        x.view(-1, w.L, w.Hkv, D)[dead] = math.nan
        c.v_pool[own] = PagedCache.to_value_layout(x)


def run(w, q, layer, new, lists=None):
    """(out, lse, the tokens that count: keys and values [s][kv])."""
    nk = w.normal(w.S, w.Hkv, D, dtype=BF16) if new else None
    nv = whole(w.S, w.g, w.Hkv, D).to(BF16).to(w.dev) if new else None
    out, lse = torch.full((w.S, w.Hq, D), math.nan, device=w.dev), torch.full((w.S, w.Hq), math.nan, device=w.dev)
    blocks = {}
    if lists is not None:
        most = max(1, max(len(x) for r in lists for x in r))
        b = torch.full((w.S, w.Hkv, most), -7, dtype=torch.int32)
        for s in range(w.S):
            for kv in range(w.Hkv):
                b[s, kv, :len(lists[s][kv])] = torch.tensor(lists[s][kv], dtype=torch.int32)
        count = torch.tensor([[len(x) for x in r] for r in lists], dtype=torch.int32)
        blocks = dict(blocks=b.to(w.dev), block_count=count.to(w.dev))
    w.md.attend(layer, q, out, new_k=nk, new_v=nv, lse=lse, **blocks)
    torch.cuda.synchronize()
    assert w.md.device_status() == 0
    tokens = []
    for s in range(w.S):
        page = w.token_pages(s)
        row = []
        for kv in range(w.Hkv):
            k, v = w.k[s][:, layer, kv], w.v[s][:, layer, kv]
            if lists is not None:
                at = torch.as_tensor(np.isin(page, lists[s][kv]))
                k, v = k[at], v[at]
            if new:
                k, v = torch.cat([k, nk[s, kv].cpu().float()[None]]), torch.cat([v, nv[s, kv].cpu().float()[None]])
            row.append((k, v))
        tokens.append(row)
    return out.cpu().double(), lse.cpu().double(), tokens


def count_tokens(w, new, lists=None):
    layer = w.L - 1
    out, lse, tokens = run(w, torch.zeros((w.S, w.Hq, D), device=w.dev), layer, new, lists)
    for s in range(w.S):
        for kv in range(w.Hkv):
            heads = slice(kv * w.G, (kv + 1) * w.G)
            v = tokens[s][kv][1]
            if v.shape[0] == 0:
                assert not out[s, heads].any() and bool((lse[s, heads] == -math.inf).all())
                continue
            ref, tol, rl, ltol = counted_bounds(v)
            assert bool(((out[s, heads] - ref).abs() <= tol).all()), (s, kv, float((out[s, heads] - ref).abs().max()))
            assert bool(((lse[s, heads] - rl).abs() <= ltol).all()), (s, kv, lse[s, heads], rl)


def drawn_lists(w, most, seed):
    rng = np.random.default_rng(seed)
    return [[sorted(rng.choice(w.pages[s], min(w.pages[s], rng.integers(0, most + 1)), replace=False).tolist()) if w.pages[s]
             else [] for _ in range(w.Hkv)] for s in range(w.S)]


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_every_token_counts_once(lens, P):
    say("[count]", lens, P)
    w = World(2, 12, 2, P, LENS[lens], seed=41)
    set_values(w, whole)
    for new in (True, False):
        count_tokens(w, new)
        for most in (1, 9, 300):
            count_tokens(w, new, drawn_lists(w, most, most))


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("aligned,quant", [(True, 0.0), (False, 0.6), (True, 0.6)])
def test_every_token_counts_once_beside_holes_and_codes(aligned, quant, P):
    say("[count]", aligned, quant, P)
    w = World(2, 12, 2, P, [700, 0, 1, 16, 2500], seed=42, aligned=aligned, quant=quant)
    set_values(w, whole)
    for new in (True, False):
        count_tokens(w, new)
        count_tokens(w, new, drawn_lists(w, 30, 5))


@pytest.mark.gpu
@pytest.mark.parametrize("shape,lens", [((1, 1, 1), [(7 * i) % 40 for i in range(1024)]),
                                        ((1, 6, 2), [(11 * i) % 70 for i in range(1024)]),
                                        ((1, 6, 2), [(131 * i) % 977 for i in range(1024)]),
                                        ((1, 16, 16), [(5 * i) % 33 for i in range(140)]),
                                        ((1, 12, 2), [(37 * i) % 211 for i in range(300)]),
                                        ((1, 2, 1), [131072 - 5]), ((1, 12, 2), [65536, 9000]),
                                        ((1, 8, 8), [32768, 32767, 32769, 31, 4097]), ((1, 16, 2), [1700] * 32)],
                         ids=["1024x1", "1024x2", "1024x2long", "140x16", "300x2", "131k", "66k+9k", "8x32k", "32x1700"])
def test_every_token_counts_once_in_the_widest_and_longest(shape, lens):
    say("[count]", shape, len(lens))
    w = World(*shape, 16, lens, seed=43, extra=0)
    set_values(w, whole)
    for new in (True, False):
        count_tokens(w, new)
        count_tokens(w, new, drawn_lists(w, 40, 6))


@pytest.mark.gpu
@pytest.mark.parametrize("new", [False, True])
@pytest.mark.parametrize("G", [1, 4, 16])
def test_bits_of_weights_and_queries(G, new):
    # two cached tokens in a tile, or one and the new token
    say("[pair]", G, new)
    S, n = 64, 1 if new else 2
    w = World(1, G, 1, 16, [n] * S, seed=44)
    k, v = torch.zeros((n, 1, 1, D)), torch.ones((n, 1, 1, D))
    k[0, ..., 0] = 1
    v[1:] = -1
    for s in range(S):
        w.cache.load_session(s, k, [1] * n, [int(w.cache.page_table[s, 0])], budget=n, clock=n)
        w.cache.load_values(s, v)
    a = pair_inputs(w.g, S, G)
    q = torch.zeros((S, G, D))
    q[:, :, 0] = a
    out, lse = torch.zeros((S, G, D), device=w.dev), torch.zeros((S, G), device=w.dev)
    token = dict(new_k=torch.zeros((S, 1, D), dtype=BF16, device=w.dev), new_v=-torch.ones((S, 1, D), dtype=BF16, device=w.dev))
    w.md.attend(0, q.to(w.dev), out, lse=lse, **(token if new else {}))
    torch.cuda.synchronize()
    ref, rl = pair_exact(a)
    tol, ltol = pair_bounds()
    err = (out.cpu().double().view(-1, D) - ref).abs().amax(1)
    say("   off by", float(err.max()) / U, "u")
    assert float(err.max()) <= tol
    lerr = (lse.cpu().double().flatten() - rl).abs()
    assert bool((lerr <= torch.tensor([ltol(float(x)) for x in rl])).all()), float(lerr.max()) / U


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[450], [1700, 3, 640, 0, 5000], [20011], [300] * 60])
def test_drawn_inputs(lens):
    say("[drawn]", len(lens))
    w = World(1, 12, 2, 16, lens, seed=45)
    for new, lists in ((True, None), (False, None), (True, drawn_lists(w, 60, 7))):
        q = w.normal(w.S, w.Hq, D) * 2
        out, lse, tokens = run(w, q, 0, new, lists)
        for s in range(w.S):
            for kv in range(w.Hkv):
                heads = slice(kv * w.G, (kv + 1) * w.G)
                k, v = tokens[s][kv]
                if k.shape[0] == 0:
                    continue
                ref, tol, rl, ltol = drawn_bounds(q[s, heads].cpu(), k, v)
                assert bool(((out[s, heads] - ref).abs() <= tol).all()), (s, kv, float(((out[s, heads] - ref).abs() / tol).max()))
                assert bool(((lse[s, heads] - rl).abs() <= ltol).all()), (s, kv)
