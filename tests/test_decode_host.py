"""The decode operators on the host: the arguments' layout, calls without a
handle, the value pool's layout, and the 64-bit oracle against closed forms
and brute force."""
import ctypes
import itertools
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import decode_oracle as O
from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import PagedCache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_argument_structs_match_the_header(tmp_path):
    structs = (B.md_rope_args, B.md_attend_args, B.md_select_args)
    lines = [f'printf("%zu\\n", sizeof({s.__name__}));' for s in structs]
    lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for s in structs for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"memdecay.h\"\nint main(void) {" + "".join(lines) +
                   "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    want = [ctypes.sizeof(s) for s in structs] + [getattr(s, f).offset for s in structs for f, _ in s._fields_]
    assert [int(x) for x in out] == want
    # packed as bytes: the same fields at the same places
    for st, packed in zip(structs, (B.ROPE_ARGS, B.ATTEND_ARGS, B.SELECT_ARGS)):
        assert packed.size == ctypes.sizeof(st) and len(st._fields_) == len(packed.unpack(bytes(packed.size)))
        for i, (name, kind) in enumerate(st._fields_):
            one = st.from_buffer_copy(packed.pack(*[1 if j == i else 0 for j in range(len(st._fields_))]))
            assert getattr(one, name) == 1 and [f for f, _ in st._fields_ if getattr(one, f)] == [name]


def test_calls_without_a_handle_are_refused():
    lib = B.load_library()
    n = ctypes.c_uint64(0)
    assert lib.md_norm_rope(None, ctypes.byref(B.md_rope_args())) == B.MD_E_INVALID
    assert lib.md_append_values(None, 0x1000, 0x1000) == B.MD_E_INVALID
    assert lib.md_attend_token(None, 0, ctypes.byref(B.md_attend_args())) == B.MD_E_INVALID
    assert lib.md_key_bounds(None, 0, 0x1000, 0x1000) == B.MD_E_INVALID
    assert lib.md_select_blocks(None, 0, ctypes.byref(B.md_select_args())) == B.MD_E_INVALID
    assert lib.md_decode_workspace(None, ctypes.byref(n), ctypes.byref(n)) == B.MD_E_INVALID


@pytest.mark.parametrize("P", [16, 64])
def test_value_layout_matches_the_header(P):
    m, L, Hkv, d = 2, 3, 2, 128
    v = torch.arange(m * P * L * Hkv * d, dtype=torch.float64).view(m, P, L, Hkv, d)
    pool = PagedCache.to_value_layout(v)
    flat = pool.reshape(m, L, Hkv, P * d)
    t, e = torch.arange(P)[:, None], torch.arange(d)[None]
    at = (t & ~15) * d + e // 32 * 512 + t // 4 % 4 * 128 + e % 16 * 8 + e // 16 % 2 * 4 + t % 4
    assert torch.equal(flat[1, 2, 1][at], v[1, :, 2, 1]) and torch.equal(flat[0, 0, 0][at], v[0, :, 0, 0])
    assert sorted(at.flatten().tolist()) == list(range(P * d))
    assert torch.equal(PagedCache.from_value_layout(pool), v)


def test_oracle_attention():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 128), (50, 128), (50, 128)))
    out, lse = O.attend(q, k, v)
    # (about 100 roundings of 2^-53 in values of at most 5 each, which may
    # cancel in the sum: 6e-14 absolute)
    for h in range(3):   # one token at a time, in order
        w = [math.exp(float(q[h] @ k[i]) / math.sqrt(128)) for i in range(50)]
        np.testing.assert_allclose(out[h], sum(a * v[i] for i, a in enumerate(w)) / math.fsum(w), rtol=1e-12, atol=1e-13)
        assert abs(float(lse[h]) - math.log(math.fsum(w))) < 1e-12
    same, l1 = O.attend(q, k[:1].expand(7, 128), v[:7])   # equal keys: the plain mean
    np.testing.assert_allclose(same, v[:7].mean(0).expand(3, 128), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(l1, q @ k[0] / math.sqrt(128) + math.log(7), rtol=1e-12)
    none, l0 = O.attend(q, k[:0], v[:0])
    assert not none.any() and (l0 == -math.inf).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotation(interleaved):
    g = torch.Generator().manual_seed(2)
    x = torch.randn((4, 2, 128), generator=g, dtype=torch.float64)
    inv = torch.as_tensor(100.0 ** (-np.arange(0, 64, 2) / 64))
    p0, p1 = torch.tensor([0, 5, 9, 100]), torch.tensor([3, 8, 12, 103])
    a, b = O.norm_rope(x, None, 0.0, p0, inv, interleaved), O.norm_rope(x, None, 0.0, p1, inv, interleaved)
    assert torch.equal(a[0], x[0]) and torch.equal(a[..., 64:], x[..., 64:])     # position 0; elements that do not turn
    np.testing.assert_allclose(a.norm(dim=-1), x.norm(dim=-1), rtol=1e-12)       # lengths stay
    y = torch.randn((1, 1, 128), generator=g, dtype=torch.float64)               # products see distances only
    c = [float((O.norm_rope(x[:1], None, 0.0, torch.tensor([p]), inv, interleaved) *
                O.norm_rope(y, None, 0.0, torch.tensor([p + 7]), inv, interleaved)).sum()) for p in (0, 50)]
    assert abs(c[0] - c[1]) < 1e-9
    w = torch.full((128,), 2.0, dtype=torch.float64)
    n = O.norm_rope(x, w, 0.0, p1, None, interleaved)
    np.testing.assert_allclose((n * n).mean(-1), np.full((4, 2), 4.0), rtol=1e-12)
    assert b.shape == x.shape


def test_oracle_bounds_hold_and_are_tight():
    rng = np.random.default_rng(3)
    for scale in (1e-6, 1.0, 3e4):
        k = rng.normal(size=(16, 128)) * scale
        lo, hi, e = O.bounds(k)
        u = 2.0 ** e
        assert (lo * u <= k.min(0)).all() and (hi * u >= k.max(0)).all()
        assert ((lo + 1) * u > k.min(0)).all() and ((hi - 1) * u < k.max(0)).all()
        assert 63 < max(np.abs(lo).max(), np.abs(hi).max()) <= 127
    assert O.bounds(np.zeros((2, 128)))[2] == O.MIN_EXP
    assert O.step_exp(127.0) == 0 and O.step_exp(127.0000001) == 1 and O.step_exp(63.5) == -1
    assert O.step_exp(1e38 * 3) == O.MAX_EXP


def test_oracle_score_bounds_the_logits():
    # whole queries that need no rounding: no key inside the bounds beats the score
    rng = np.random.default_rng(4)
    for _ in range(20):
        k, q = rng.integers(-127, 128, (16, 128)), rng.integers(-127, 128, (2, 128))
        q[:, 0] = 127
        lo, hi, e = O.bounds(k)
        s = O.block_score(q, lo, hi, e)
        assert s >= (k @ q.T).max()
        corner = np.where(q[0] > 0, hi, lo) * 2.0 ** e
        assert s >= corner @ q[0]
    small = np.zeros((1, 128))
    small[0, :3] = [127, -127, 1]
    lo, hi = np.zeros(128, np.int64), np.zeros(128, np.int64)
    lo[:3], hi[:3] = [-2, -3, -4], [2, 3, 4]
    best = max(a * 127 - b * 127 + c for a, b, c in itertools.product((-2, 2), (-3, 3), (-4, 4)))
    assert O.block_score(small, lo, hi, 0) == best


def test_oracle_selection():
    assert O.select([1.0, 5.0, 5.0, 2.0, 9.0], 2, 0, 0) == [1, 4]           # ties to the older page
    assert O.select([1.0, 5.0, 5.0, 2.0, 9.0], 3, 1, 1) == [0, 1, 4]
    assert O.select([1.0, 5.0], 2, 0, 0) == [0, 1] and O.select([], 3, 1, 1) == []
    assert O.select([0.0, -math.inf, -1.0], 2, 0, 0) == [0, 2]


def test_values_go_where_the_sessions_keys_are():
    # more or fewer tokens than the session holds would reach pages that it
    # lacks (or leave some without values): refused before anything is written
    c = PagedCache(L=1, Hq=2, Hkv=1, d=128, P=16, S=2, max_pages=4, n_phys=6, device="cpu", values=True)
    keys = torch.zeros((20, 1, 1, 128), dtype=torch.bfloat16)
    c.load_session(0, keys, [1] * 20, [4, 2], budget=20, clock=20)
    c.v_pool.zero_()
    for n in (1, 19, 21, 33, 64, 100):
        with pytest.raises(ValueError):
            c.load_values(0, torch.ones((n, 1, 1, 128), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        c.load_values(1, keys)                 # a session without pages
    with pytest.raises(ValueError):
        c.load_values(0, keys, [1] * 10 + [2] * 10)   # its keys lie without holes
    assert int(torch.count_nonzero(c.v_pool)) == 0
    values = torch.arange(20 * 128).to(torch.bfloat16).view(20, 1, 1, 128)
    c.load_values(0, values)
    got = c.from_value_layout(c.v_pool[torch.tensor([4, 2])]).reshape(32, 1, 1, 128)
    assert torch.equal(got[:20], values) and int(torch.count_nonzero(got[20:])) == 0
    with pytest.raises(ValueError):
        PagedCache(L=1, Hq=2, Hkv=1, d=128, P=16, S=1, max_pages=4, n_phys=4, device="cpu").load_values(0, keys)
