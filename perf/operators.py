"""Cases of a decode engine's operators around the paged cache: preparing a
token's heads, attending over the cache, and picking the pages to attend to.

A case's ``op`` says which operator a pass calls:

  rope    norms of the query and key heads of fused projection rows with the
          rotation by position in the same pass; the values go along
  attend  attention of one new token of every session, in one layer, over the
          session's pages and the token itself
  sparse  the same over a list of pages per session and KV head
  bounds  lower and upper bounds of the keys of a page, in 8 bits: of every
          page (after the prompts) or of each session's last (every step)
  select  the pages whose bounds promise the largest logits, per session and
          KV head

``quant``: share of pages holding 8-bit keys; ``aligned``: region-aligned
pages, whose unused slots are holes.  Sizes are those of synth/configs.py and
of the GPU tests, and one generic grouped-query shape with eight KV heads.

Where ``own`` is false, ``run`` computes the operators in elementary torch
operations; where it is true, through the package's calls.
"""
import math

import numpy as np
import torch

own = False

HEAD = 128
HOLE = 255
SINK, RECENT = 1, 2        # pages a selection always takes: the first, the newest
EPS = 1e-6
THETA = 1000000.0
EXP_MIN, EXP_MAX = -100, 100
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rope(name, rows, L, Hq, Hkv, **kw):
    return dict(dict(name=name, op="rope", T=rows, L=L, Hq=Hq, Hkv=Hkv, type="bf16", norm=True, rot=HEAD, pairs=False,
                     far=65536, decode=False), **kw)


def _cache_case(name, op, L, Hq, Hkv, P, S, lo, hi, **kw):
    return dict(dict(name=name, op=op, L=L, Hq=Hq, Hkv=Hkv, P=P, S=S, lo=lo, hi=hi, quant=0.0, aligned=False, out="bf16",
                     token=True, blocks=0, all=False), **kw)


def listed():
    return [
        # one decode step of a batch of agent episodes: a row per session, latency counts
        _rope("rope_step_32", 32, 36, 16, 2, decode=True),
        # a long prompt's rows of one layer, into the layout the prompt's keys are kept in
        _rope("rope_prompt_32k", 32768, 28, 12, 2),
        # the smallest call: one layer of one short chat
        _cache_case("attend_1x450", "attend", 1, 12, 2, 16, 1, 450, 450),
        # one layer of a batch of agent episodes (3B shape)
        _cache_case("attend_32x1700", "attend", 36, 16, 2, 16, 32, 1700, 1700),
        # a large serving batch of uneven sessions, pages of 64
        _cache_case("attend_64_ragged", "attend", 4, 16, 2, 64, 64, 2048, 65536),
        # long-horizon sessions, most of their pages in the 8-bit tier
        _cache_case("attend_16x32k_quant", "attend", 28, 12, 2, 16, 16, 32768, 32768, quant=0.75, out="f32"),
        # long-horizon sessions attending to 256 of their 2,048 pages
        _cache_case("sparse_16x32k", "sparse", 28, 12, 2, 16, 16, 32768, 32768, blocks=256),
        # one session at the largest page table, attending to 512 of 8,192 pages
        _cache_case("sparse_1x131k", "sparse", 4, 32, 8, 16, 1, 131071, 131071, blocks=512),
        # every step: the bounds of the pages that took a token
        _cache_case("bounds_step_32x1700", "bounds", 36, 16, 2, 16, 32, 1700, 1700),
        # once after the prompts: the bounds of every page
        _cache_case("bounds_prompt_16x32k", "bounds", 28, 12, 2, 16, 16, 32768, 32768, all=True),
        # picking 128 pages for a large batch of uneven sessions
        _cache_case("select_64_ragged", "select", 4, 16, 2, 16, 64, 2048, 65536, blocks=128),
        # picking pages for one session at the largest page table
        _cache_case("select_1x131k", "select", 4, 32, 8, 16, 1, 131071, 131071, blocks=512),
    ]


MOST_BYTES = 7.9e9        # of a drawn case's pass, and
MOST_POOL = 9.0e9         # of a drawn case's keys in all its layers


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    shapes = [(1, 12, 2), (28, 12, 2), (36, 16, 2), (4, 32, 8), (2, 16, 1), (3, 5, 5)]
    while True:
        op = rng.choice(["rope", "attend", "attend", "sparse", "bounds", "select"])
        L, Hq, Hkv = rng.choice(shapes)
        if op == "rope":
            decode = rng.random() < 0.4
            c = _rope(None, log_int(1, 512) if decode else log_int(16, 32768), L, Hq, Hkv,
                      type=rng.choice(["bf16", "bf16", "f16", "f32"]), norm=rng.random() < 0.7,
                      rot=rng.choice([HEAD, HEAD, 64, 32]), pairs=rng.random() < 0.3, far=log_int(1000, 4000000),
                      decode=decode)
            del c["name"]
            return c
        P = rng.choice([16, 16, 64])
        S, hi = log_int(1, 64), log_int(1 if op != "bounds" else 17, 131072 - 16)
        lo = max(1, hi // rng.choice([1, 1, 3, 16]))
        c = _cache_case(None, op, L, Hq, Hkv, P, S, lo, hi)
        del c["name"]
        if op in ("attend", "sparse"):
            c["quant"] = rng.choice([0.0, 0.0, 0.75])
            c["aligned"] = rng.random() < 0.2
            c["out"] = rng.choice(["bf16", "f32"])
            c["token"] = rng.random() < 0.8
        if op in ("sparse", "select"):
            c["blocks"] = log_int(SINK + RECENT + 1, 512)
            if op == "select" and 3 * c["blocks"] > 2 * max(_pages(c)):   # there is something to pick from
                continue
        if op == "bounds":
            c["all"] = rng.random() < 0.5
            c["aligned"] = rng.random() < 0.2
        pool = sum(_pages(c)) * P * L * Hkv * HEAD * 2
        padded = S * max(_pages(c)) * P * Hkv * HEAD * 4   # the plain form's keys of one layer
        if work(c)["bytes"] <= MOST_BYTES and pool <= MOST_POOL and padded <= 6e9:
            return c


# ------------------------------------------------------------------ inputs

def _lengths(c):
    """Slots in use of each session, spread evenly over [lo, hi] in a
    scattered order (the same for every seed, so that a case's work is fixed)."""
    lo, hi, S = c["lo"], c["hi"], c["S"]
    return [int(lo + (hi - lo) * ((0.618033988749895 * (s + 1)) % 1.0)) if lo < hi else lo for s in range(S)]


def _pages(c):
    return [-(-n // c["P"]) for n in _lengths(c)]


def _gen(seed, *at):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence([seed, *at]).generate_state(1, np.uint64)[0] >> 1))
    return g


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _tables(c, seed):
    """Lengths and page tables, pages scattered over the pool."""
    rng = np.random.default_rng([seed, 3])
    n, m = np.array(_lengths(c)), np.array(_pages(c))
    most = int(m.max()) + (1 if int(m.max()) < 8192 else 0)   # room for a page more
    NP = int(m.sum()) + c["S"] + 3
    ids = rng.permutation(NP).astype(np.int32)
    table = np.full((c["S"], most), -1, np.int32)
    ends = np.cumsum(m)
    for s in range(c["S"]):
        table[s, :m[s]] = ids[ends[s] - m[s]:ends[s]]
    region = rng.integers(0, 7, (NP, c["P"])).astype(np.uint8)
    if c["aligned"]:   # a third of the pages were closed early
        live = np.where(rng.random(NP) < 0.33, rng.integers(1, c["P"] + 1, NP), c["P"])
        region[np.arange(c["P"])[None, :] >= live[:, None]] = HOLE
        for s in range(c["S"]):   # the last slot in use holds a token
            last = region[table[s, m[s] - 1]]
            last[:n[s] - (m[s] - 1) * c["P"]][last[:n[s] - (m[s] - 1) * c["P"]] == HOLE] = 1
    return n, m, table, region, rng


def _pool_keys(c, seed, NP):
    """Keys in the pool's layout [NP][L][Hkv][P/16][d/8][16][8]: a direction
    that the tokens of a page share, noise, and a few tokens that draw
    attention."""
    L, Hkv, nb = c["L"], c["Hkv"], c["P"] // 16
    out = torch.empty((NP, L, Hkv, nb, 16, 16, 8), dtype=torch.bfloat16, device="cuda")
    step = max(1, 2 ** 26 // (L * Hkv * nb * 2048))
    for i, part in enumerate(out.split(step)):
        g = _gen(seed, 1, i)
        k = len(part)
        scale = torch.rand((k, 1, 1, nb, 1, 16, 1), generator=g, device="cuda") + 0.4
        scale = torch.where(torch.rand(scale.shape, generator=g, device="cuda") < 0.02, 2.0, scale)
        x = _normal(g, k, L, Hkv, nb, 16, 16, 8).mul_(0.8).add_(_normal(g, k, L, Hkv, 1, 16, 1, 8), alpha=0.6)
        part.copy_(x.mul_(scale))
    return out


def _pool_values(c, seed, NP):
    """Values in the pool's layout [NP][L][Hkv][P/16][d/32][4][16][2][4]."""
    out = torch.empty((NP, c["L"], c["Hkv"], c["P"] // 16, 4, 4, 16, 2, 4), dtype=torch.bfloat16, device="cuda")
    for i, part in enumerate(out.split(max(1, 2 ** 27 // (out[0].numel())))):
        part.normal_(generator=_gen(seed, 2, i))
    return out


def _write_codes(c, pool, ids):
    """Turn pages into the 8-bit tier's layout: per 16-token block the codes
    in the order [e / 64][(e / 8) % 4][t][(e / 32) % 2][e % 8], the scale
    four times at byte 2048."""
    for part in ids.split(256):
        x = pool[part].float().permute(0, 1, 2, 3, 5, 4, 6).reshape(-1, 16, HEAD)   # [block][t][e]
        scale = x.abs().amax(dim=(1, 2)) / 448.0
        codes = (x / scale[:, None, None]).to(torch.float8_e4m3fn)
        raw = torch.zeros((x.shape[0], 4096), dtype=torch.uint8, device="cuda")
        raw[:, :2048] = codes.view(torch.uint8).view(-1, 16, 2, 2, 4, 8).permute(0, 2, 4, 1, 3, 5).reshape(-1, 2048)
        raw[:, 2048:2064] = scale.view(-1, 1).repeat(1, 4).view(torch.uint8)
        pool[part] = raw.view(torch.bfloat16).view(pool[part].shape)


def _prepare_rope(c, seed):
    T, Hq, Hkv, L = c["T"], c["Hq"], c["Hkv"], c["L"]
    g = _gen(seed, 5)
    rng = np.random.default_rng([seed, 6])
    st = dict(case=c)
    wide = (Hq + 2 * Hkv) * HEAD
    st["qkv"] = _normal(g, T, wide).mul_(torch.rand((T, 1), generator=g, device="cuda") * 4 + 0.1).to(TYPES[c["type"]])
    st["w"] = [torch.rand(HEAD, generator=g, device="cuda") + 0.5 for _ in range(2)] if c["norm"] else [None, None]
    st["inv_freq"] = torch.as_tensor(THETA ** (-np.arange(0, c["rot"], 2) / c["rot"]), device="cuda")
    if c["decode"]:   # each session's next position: its clock
        st["position"] = torch.as_tensor(rng.integers(0, c["far"], T).astype(np.int32), device="cuda")
    else:
        st["position"] = torch.arange(T, dtype=torch.int32, device="cuda") + int(rng.integers(0, c["far"]))
    # a step's query buffer and new keys hold every layer, a prompt's keys one at a time
    layers = L if c["decode"] else 1
    st["q_out"] = torch.empty((T, layers, Hq, HEAD), device="cuda")
    st["k_out"] = torch.empty((T, layers, Hkv, HEAD), dtype=torch.bfloat16, device="cuda")
    st["v_out"] = torch.empty((T, layers, Hkv, HEAD), dtype=torch.bfloat16, device="cuda")
    return st


def prepare(case, seed):
    c = case
    if c["op"] == "rope":
        st = _prepare_rope(c, seed)
        if own:
            st["md"] = _handle(dict(c, P=16, S=c["T"] if c["decode"] else 1, quant=0.0, aligned=False, op="rope"), st)
        return st
    S, L, Hq, Hkv = c["S"], c["L"], c["Hq"], c["Hkv"]
    n, m, table, region, rng = _tables(c, seed)
    NP = len(region)
    st = dict(case=c, layer=L // 2, most=int(m.max()))
    for name, x in (("n_tokens", n), ("n_pages", m), ("page_table", table), ("region", region)):
        st[name] = torch.as_tensor(x if name == "region" else x.astype(np.int32), device="cuda")
    st["page_format"] = torch.zeros(NP, dtype=torch.uint8, device="cuda")
    g = _gen(seed, 4)
    st["q"] = _normal(g, S, Hq, HEAD)
    if c["op"] != "select":
        st["k_pool"] = _pool_keys(c, seed, NP)
    if c["op"] in ("attend", "sparse"):
        st["v_pool"] = _pool_values(c, seed, NP)
        st["new_k"] = _normal(g, S, Hkv, HEAD).to(torch.bfloat16) if c["token"] else None
        st["new_v"] = _normal(g, S, Hkv, HEAD).to(torch.bfloat16) if c["token"] else None
        st["out"] = torch.empty((S, Hq, HEAD), dtype=TYPES[c["out"]], device="cuda")
        st["lse"] = torch.empty((S, Hq), device="cuda")
        if c["quant"] > 0:
            full = torch.as_tensor(rng.permutation(np.concatenate([table[s, :m[s] - 1] for s in range(S)])), device="cuda")
            ids = full[:int(c["quant"] * len(full))].long()
            _write_codes(c, st["k_pool"], ids)
            st["page_format"][ids] = 1
    if c["op"] == "bounds":   # one row more, where the plain form's padding goes
        st["bounds"] = torch.zeros((NP + 1, L, Hkv, 2, HEAD), dtype=torch.int8, device="cuda")
        st["exp"] = torch.zeros((NP + 1, L, Hkv), dtype=torch.int8, device="cuda")
    if c["op"] == "select":
        mid = _normal(g, NP, L, Hkv, 1, HEAD).mul_(24)
        half = torch.rand((NP, L, Hkv, 1, HEAD), generator=g, device="cuda") * 50 + 20
        st["bounds"] = torch.cat([mid - half, mid + half], dim=3).round_().clamp_(-127, 127).to(torch.int8)
        st["exp"] = torch.randint(-7, -4, (NP, L, Hkv), generator=g, device="cuda").to(torch.int8)
    if c["op"] in ("sparse", "select"):
        st["blocks"] = torch.full((S, Hkv, c["blocks"]), -1, dtype=torch.int32, device="cuda")
        st["count"] = torch.zeros((S, Hkv), dtype=torch.int32, device="cuda")
    if c["op"] == "sparse":
        b, k = _lists(c, m, rng)
        st["blocks"].copy_(torch.as_tensor(b))
        st["count"].copy_(torch.as_tensor(k))
    if own:
        st["md"] = _handle(c, st)
    return st


def _lists(c, m, rng):
    """Ascending lists of pages as a selection leaves them: the first page,
    the newest, and others in scattered runs."""
    b = np.full((c["S"], c["Hkv"], c["blocks"]), -1, np.int32)
    count = np.minimum(m, c["blocks"])[:, None].repeat(c["Hkv"], 1).astype(np.int32)
    for s in range(c["S"]):
        forced = np.unique(np.concatenate([np.arange(min(SINK, m[s])), np.arange(max(0, m[s] - RECENT), m[s])]))
        rest = np.setdiff1d(np.arange(m[s]), forced)
        for kv in range(c["Hkv"]):
            k = count[s, kv]
            more = rng.choice(rest, k - len(forced), replace=False) if k > len(forced) else rest[:0]
            b[s, kv, :k] = np.sort(np.concatenate([forced, more]))[:k]
    return b, count


def _handle(c, st):
    """The program's cache and handle, on the tensors of the state."""
    from paper_2607_10582_amd.cache import MemDecay, PagedCache
    pool = st.get("k_pool")
    NP = len(st["region"]) if "region" in st else 1
    MP = st["page_table"].shape[1] if "page_table" in st else 1
    shape = dict(L=c["L"], Hq=c["Hq"], Hkv=c["Hkv"], d=HEAD, P=c["P"], S=c["S"])
    cache = PagedCache(**shape, max_pages=MP, n_phys=NP if pool is None else 1)
    cache.n_phys = NP
    for name in ("k_pool", "v_pool", "region", "n_tokens", "n_pages", "page_table", "page_format"):
        if name in st:
            setattr(cache, name, st[name])
    if "n_tokens" in st:
        cache.n_live = st["n_tokens"].clone()
        cache.budget.copy_(st["n_tokens"])
        for name in ("t_ins", "t_ref"):
            setattr(cache, name, torch.zeros((NP, c["P"]), dtype=torch.int32, device="cuda"))
        cache.importance = torch.zeros((NP, c["P"]), device="cuda")
        cache.free_list = torch.zeros(NP, dtype=torch.int32, device="cuda")
    if "bounds" in st:
        cache.key_bounds, cache.bound_exp = st["bounds"][:NP], st["exp"][:NP]
    if "position" in st and c["op"] == "rope" and len(st["position"]) == c["S"]:
        cache.clock.copy_(st["position"])
    ones = torch.ones((c["S"], 7))
    return MemDecay(cache, ones, ones, rho=0.9, alpha=1.0, tau_scale=2.0, pinned_mask=1, fused=True,
                    region_aligned=c["aligned"], quant_threshold=0.3 if c["quant"] > 0 else 0.0)


# ------------------------------------------------------------------ a pass

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    c, md = st["case"], st["md"]
    op = c["op"]
    if op == "rope":
        q, k, v = (st[x][:, c["L"] // 2 if c["decode"] else 0] for x in ("q_out", "k_out", "v_out"))
        md.norm_rope(st["qkv"], q, k, v, q_weight=st["w"][0], k_weight=st["w"][1], eps=EPS, inv_freq=st["inv_freq"],
                     position=None if c["decode"] else st["position"], interleaved=c["pairs"])
        return dict(q=q, k=k, v=v)
    if op in ("attend", "sparse"):
        lists = dict(blocks=st["blocks"], block_count=st["count"]) if op == "sparse" else {}
        md.attend(st["layer"], st["q"], st["out"], new_k=st["new_k"], new_v=st["new_v"], lse=st["lse"], **lists)
        return dict(out=st["out"], lse=st["lse"])
    if op == "bounds":
        md.update_bounds(all_pages=c["all"])
        return dict(bounds=st["bounds"][:-1], exp=st["exp"][:-1])
    md.select_blocks(st["layer"], st["q"], st["blocks"], st["count"], first=SINK, last=RECENT)
    return dict(blocks=st["blocks"], count=st["count"])


def _run_plain(st):
    op = st["case"]["op"]
    return {"rope": _plain_rope, "attend": _plain_attend, "sparse": _plain_attend, "bounds": _plain_bounds,
            "select": _plain_select}[op](st)


def _plain_rope(st):
    c = st["case"]
    T, Hq, Hkv, r = c["T"], c["Hq"], c["Hkv"], c["rot"]
    x = st["qkv"].view(T, Hq + 2 * Hkv, HEAD)
    q, k, v = x.split([Hq, Hkv, Hkv], dim=1)

    def normed(x, w):
        return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w

    q, k = normed(q.float(), st["w"][0]), normed(k.float(), st["w"][1])
    angle = (st["position"].double()[:, None] * st["inv_freq"])[:, None]   # positions far out need 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(x):
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["pairs"] else (x[..., :r // 2], x[..., r // 2:r])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.stack([a, b], -1).flatten(-2) if c["pairs"] else torch.cat([a, b], -1)
        return torch.cat([y, x[..., r:]], -1)

    return dict(q=turned(q), k=turned(k).to(torch.bfloat16), v=v.to(torch.bfloat16))


def _widen(k, fmt):
    """Keys of pages [..][P/16][d/8][16][8] -> [..][P/16][16][d] in 32 bits;
    fmt [..]: 1 where the page holds codes and scales."""
    plain = k.float().transpose(-2, -3).flatten(-2)
    if fmt is None:
        return plain
    raw = k.flatten(-3).view(torch.uint8)
    codes = raw[..., :2048].contiguous().view(torch.float8_e4m3fn).float()
    codes = codes.unflatten(-1, (2, 4, 16, 2, 8)).movedim(-3, -5).transpose(-3, -2)   # [t][e/64][(e/32)%2][(e/8)%4][e%8]
    scale = raw[..., 2048:2052].contiguous().view(torch.float32)
    return torch.where(fmt[..., None, None, None].bool(), codes.flatten(-4) * scale[..., None], plain)


def _plain_attend(st):
    c = st["case"]
    S, Hkv, P = c["S"], c["Hkv"], c["P"]
    G, layer = c["Hq"] // Hkv, st["layer"]
    every = st["page_table"][:, :st["most"]].clamp(min=0).long()
    if c["op"] == "sparse":
        at = st["blocks"].clamp(min=0).long()                       # [S][Hkv][pages]
        given = st["blocks"] >= 0
        page = every.gather(1, at.flatten(1)).view(at.shape)
    else:
        at = torch.arange(st["most"], device="cuda").expand(S, Hkv, -1)
        given = at < st["n_pages"][:, None, None]
        page = every[:, None].expand(-1, Hkv, -1)
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    fmt = st["page_format"][page] if c["quant"] > 0 else None
    k = _widen(st["k_pool"][page, layer, head], fmt).reshape(S, Hkv, -1, HEAD)
    # values [P/16][d/32][4][16][2][4]: token 4 g + j, dim 32 b + 16 i + e
    v = st["v_pool"][page, layer, head].float().permute(0, 1, 2, 3, 5, 8, 4, 7, 6).reshape(S, Hkv, -1, HEAD)
    slot = at[..., None] * P + torch.arange(P, device="cuda")
    seen = given[..., None] & (slot < st["n_tokens"][:, None, None, None])
    if c["aligned"]:
        seen = seen & (st["region"][page] != HOLE)
    seen = seen.flatten(2)
    v = v * seen[..., None]
    if st["new_k"] is not None:
        k = torch.cat([k, st["new_k"].float()[:, :, None]], 2)
        v = torch.cat([v, st["new_v"].float()[:, :, None]], 2)
        seen = torch.cat([seen, torch.ones_like(seen[..., :1])], 2)
    x = torch.matmul(st["q"].view(S, Hkv, G, HEAD), k.transpose(2, 3)) / math.sqrt(HEAD)
    x = x.masked_fill(~seen[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e, v) / total
    lse = (top + total.log()).flatten(1)
    return dict(out=out.view(S, -1, HEAD).to(st["out"].dtype), lse=lse)


def _power(e):
    return ((e.int() + 127) << 23).view(torch.float32)   # 2^e


def _step_exp(amax):
    """The least e in [EXP_MIN, EXP_MAX] with amax <= 127 * 2^e."""
    f, e = torch.frexp(amax)
    return torch.where(amax > 0, e - 7 + (f > 127 / 128), EXP_MIN).clamp(EXP_MIN, EXP_MAX)


def _plain_bounds(st):
    c = st["case"]
    P, NP = c["P"], st["bounds"].shape[0] - 1
    last = st["n_pages"][:, None].long() - 1
    at = torch.arange(st["most"], device="cuda").expand(c["S"], -1) if c["all"] else last
    page = st["page_table"].long().gather(1, at)
    slot = at[..., None] * P + torch.arange(P, device="cuda")
    seen = slot < st["n_tokens"][:, None, None]
    if c["aligned"]:
        seen = seen & (st["region"][page.clamp(min=0)] != HOLE)
    page = torch.where(at <= last, page, NP).flatten()
    seen = seen.flatten(0, 1).view(len(page), 1, 1, -1, 1, 16, 1)
    k = st["k_pool"][page.clamp(max=NP - 1)].float()
    hi = k.masked_fill(~seen, -math.inf).amax((3, 5)).flatten(3)    # [page][L][Hkv][d]
    lo = k.masked_fill(~seen, math.inf).amin((3, 5)).flatten(3)
    e = _step_exp(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    unit = _power(-e)[..., None]
    both = torch.stack([torch.floor(lo * unit), torch.ceil(hi * unit)], 3).clamp(-127, 127)
    st["bounds"][page] = both.to(torch.int8)
    st["exp"][page] = e.to(torch.int8)
    return dict(bounds=st["bounds"][:-1], exp=st["exp"][:-1])


def _plain_select(st):
    c = st["case"]
    S, Hkv, K = c["S"], c["Hkv"], c["blocks"]
    G, m, layer = c["Hq"] // Hkv, st["most"], st["layer"]
    page = st["page_table"][:, :m].clamp(min=0).long()
    b = st["bounds"][page, layer].permute(0, 2, 1, 3, 4).float()            # [S][Hkv][m][2][d]
    e = st["exp"][page, layer].permute(0, 2, 1).int()                      # [S][Hkv][m]
    q = st["q"].view(S, Hkv, G, HEAD)
    qe = _step_exp(q.abs().amax(-1))
    code = torch.round(q * _power(-qe)[..., None])
    code = torch.cat([code.clamp(max=0), code.clamp(min=0)], -1)            # against lower, upper bounds
    dot = torch.matmul(code, b.flatten(3).transpose(2, 3))                  # whole numbers below 2^24
    score = (dot.double() * _power(qe).double()[..., None] * _power(e).double()[:, :, None]).amax(2)
    at = torch.arange(m, device="cuda")
    n = st["n_pages"][:, None, None]
    score = score.masked_fill((at < SINK) | (at >= n - RECENT), math.inf).masked_fill(at >= n, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :K]
    best = torch.where(best < n, best, m).sort(-1).values                   # pages that are not there go last
    blocks = torch.full_like(st["blocks"], -1)
    blocks[..., :best.shape[-1]] = torch.where(best < m, best, -1)
    count = st["n_pages"].clamp(max=K)[:, None].expand(S, Hkv)
    return dict(blocks=blocks, count=count.contiguous())


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once, each output written once; for the attention the
    tokens attended to, their keys as stored, and 4 d operations per query
    head and token."""
    c = case
    if c["op"] == "rope":
        size = 4 if c["type"] == "f32" else 2
        per = (c["Hq"] + 2 * c["Hkv"]) * HEAD * size + c["Hq"] * HEAD * 4 + 2 * c["Hkv"] * HEAD * 2 + 4
        return {"bytes": c["T"] * per, "flops": c["T"] * (c["Hq"] + c["Hkv"]) * HEAD * 10.0}
    S, Hq, Hkv, P, L = c["S"], c["Hq"], c["Hkv"], c["P"], c["L"]
    n, m = _lengths(c), _pages(c)
    if c["op"] in ("attend", "sparse"):
        tokens = sum(n) if c["op"] == "attend" else sum(min(x, c["blocks"] * P) for x in n)
        key = 2 - (1 - 1 / 512) * c["quant"]
        small = S * Hq * HEAD * (4 + TYPES[c["out"]].itemsize) + 4 * sum(m)
        return {"bytes": tokens * Hkv * HEAD * (key + 2) + small, "flops": 4.0 * tokens * Hq * HEAD}
    if c["op"] == "bounds":
        tokens = sum(n) if c["all"] else sum(x - (y - 1) * P for x, y in zip(n, m))
        pages = sum(m) if c["all"] else S
        return {"bytes": L * Hkv * (tokens * HEAD * 2 + pages * (2 * HEAD + 1)), "flops": 2.0 * L * Hkv * tokens * HEAD}
    pages = sum(m)
    return {"bytes": pages * (Hkv * (2 * HEAD + 1) + 4) + S * Hq * HEAD * 4 + S * Hkv * c["blocks"] * 4,
            "flops": 2.0 * pages * Hq * 2 * HEAD}


# ------------------------------------------------------------------ in 64 bits

def _exact_rope(c, seed):
    st = _prepare_rope(c, seed)
    Hq, Hkv, half = c["Hq"], c["Hkv"], c["rot"] // 2
    x = st["qkv"].double().view(c["T"], -1, HEAD)
    for lo, hi, w in ((0, Hq, st["w"][0]), (Hq, Hq + Hkv, st["w"][1])):
        if w is not None:
            x[:, lo:hi] /= ((x[:, lo:hi] ** 2).sum(-1, keepdim=True) / HEAD + EPS).sqrt()
            x[:, lo:hi] *= w.double()
    heads = x[:, :Hq + Hkv]
    first = torch.arange(half, device="cuda") * (2 if c["pairs"] else 1)
    second = first + (1 if c["pairs"] else half)
    z = torch.complex(heads[..., first], heads[..., second])
    z = z * torch.polar(torch.ones_like(st["inv_freq"]), st["position"].double()[:, None] * st["inv_freq"])[:, None]
    heads[..., first], heads[..., second] = z.real, z.imag
    return dict(q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:])


def _exact_attend(c, seed):
    st = prepare(c, seed)
    S, Hkv, P = c["S"], c["Hkv"], c["P"]
    G, layer = c["Hq"] // Hkv, st["layer"]
    n, table = st["n_tokens"].tolist(), st["page_table"].tolist()
    lists = st["blocks"].tolist() if c["op"] == "sparse" else None
    out = torch.empty((S, c["Hq"], HEAD), dtype=torch.float64, device="cuda")
    lse = torch.empty((S, c["Hq"]), dtype=torch.float64, device="cuda")
    byte = torch.arange(HEAD, device="cuda")
    byte = 1024 * (byte // 64) + 256 * ((byte // 8) % 4) + 8 * ((byte // 32) % 2) + byte % 8
    for s in range(S):
        for h in range(Hkv):
            blocks = range(-(-n[s] // P)) if lists is None else [b for b in lists[s][h] if b >= 0]
            slots = [min(P, n[s] - b * P) for b in blocks]
            ids = torch.tensor([table[s][b] for b in blocks], device="cuda")
            t = torch.arange(P, device="cuda")
            ok = t[None] < torch.tensor(slots, device="cuda")[:, None]
            if c["aligned"]:
                ok &= st["region"][ids] != HOLE
            page, t = ok.nonzero(as_tuple=True)
            kk, vv = st["k_pool"][ids, layer, h].flatten(1), st["v_pool"][ids, layer, h].flatten(1)
            e, base = torch.arange(HEAD, device="cuda"), (t // 16 * 16 * HEAD)[:, None]
            k = kk[page[:, None], base + (e // 8) * 128 + (t % 16)[:, None] * 8 + e % 8].double()
            t4 = (t % 16 // 4)[:, None]
            v = vv[page[:, None], base + e // 32 * 512 + t4 * 128 + e % 16 * 8 + e // 16 % 2 * 4 + (t % 4)[:, None]].double()
            if c["quant"] > 0:
                raw = kk.view(torch.uint8)
                code = raw[page[:, None], 2 * base + byte + 16 * (t % 16)[:, None]].view(torch.float8_e4m3fn).double()
                at = 2 * base + 2048 + torch.arange(4, device="cuda")
                scale = raw[page[:, None], at].contiguous().view(torch.float32).double()
                k = torch.where((st["page_format"][ids][page] == 1)[:, None], code * scale, k)
            if st["new_k"] is not None:
                k, v = torch.cat([k, st["new_k"][s, h].double()[None]]), torch.cat([v, st["new_v"][s, h].double()[None]])
            x = k @ st["q"][s, h * G:(h + 1) * G].double().t().contiguous() / math.sqrt(HEAD)
            z = torch.logsumexp(x, 0)
            lse[s, h * G:(h + 1) * G] = z
            out[s, h * G:(h + 1) * G] = torch.exp(x - z).t().contiguous() @ v
    return dict(out=out, lse=lse)


def exact(case, seed):
    if case["op"] == "rope":
        return _exact_rope(case, seed)
    if case["op"] in ("attend", "sparse"):
        return _exact_attend(case, seed)
    return None   # bounds and choices are whole numbers
