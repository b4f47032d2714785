"""The row operators on the host: the arguments' layout, their checks under
AddressSanitizer and UndefinedBehaviorSanitizer, the 8-bit values' layout, and
the 64-bit definitions against brute force."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2607_10582_amd import binding as B
from paper_2607_10582_amd.cache import PagedCache
from rows_world import D, attend, quantise, quantise_slots, visible

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_argument_structs_match_the_header(tmp_path):
    structs = (B.md_row_list, B.md_values, B.md_write_args, B.md_read_args, B.md_rows_args)
    lines = [f'printf("%zu\\n", sizeof({s.__name__}));' for s in structs]
    lines += [f'printf("%zu\\n", offsetof({s.__name__}, {f}));' for s in structs for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"memdecay.h\"\nint main(void) {" + "".join(lines) +
                   f'printf("%d\\n", MD_DEV_BAD_ROW); return 0; }}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    want = [ctypes.sizeof(s) for s in structs] + [getattr(s, f).offset for s in structs for f, _ in s._fields_]
    assert [int(x) for x in out] == want + [B.MD_DEV_BAD_ROW]


def leaves(struct, base=0):
    for name, kind in struct._fields_:
        at = base + getattr(struct, name).offset
        if issubclass(kind, ctypes.Structure):
            yield from leaves(kind, at)
        else:
            yield at, ctypes.sizeof(kind)


@pytest.mark.parametrize("struct,packed", [(B.md_values, B.VALUES), (B.md_write_args, B.WRITE_ARGS),
                                           (B.md_read_args, B.READ_ARGS), (B.md_rows_args, B.ROWS_ARGS)])
def test_packed_arguments_are_the_struct(struct, packed):
    fields = list(leaves(struct))
    assert packed.size == ctypes.sizeof(struct) and len(packed.unpack(bytes(packed.size))) == len(fields)
    for i, (at, size) in enumerate(fields):
        raw = packed.pack(*[1 if j == i else 0 for j in range(len(fields))])
        assert int.from_bytes(raw[at:at + size], "little") == 1 and sum(raw) == 1


def test_calls_without_a_handle_are_refused():
    lib = B.load_library()
    n = ctypes.c_uint64(0)
    assert lib.md_append_codes(None, 0x1000, ctypes.byref(B.md_values())) == B.MD_E_INVALID
    assert lib.md_write_rows(None, 0, ctypes.byref(B.md_write_args())) == B.MD_E_INVALID
    assert lib.md_read_rows(None, 0, ctypes.byref(B.md_read_args())) == B.MD_E_INVALID
    assert lib.md_attend_values(None, 0, ctypes.byref(B.md_attend_args()), ctypes.byref(B.md_values()), 0, 0) == B.MD_E_INVALID
    assert lib.md_attend_rows(None, 0, ctypes.byref(B.md_rows_args())) == B.MD_E_INVALID
    assert lib.md_rows_workspace(None, ctypes.byref(n)) == B.MD_E_INVALID


def test_arguments_under_sanitizers(tmp_path):
    exe = tmp_path / "rows_args"
    # (what the checks do not reach, the other launchers and the HIP runtime, stays unresolved)
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "rows_args.cpp"),
           "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "passed under the sanitizers" in r.stdout


@pytest.mark.parametrize("P", [16, 64])
def test_code_layout_matches_the_header(P):
    m, L, Hkv = 2, 3, 2
    v = torch.randn((m, P, L, Hkv, D), generator=torch.Generator().manual_seed(1)).bfloat16()
    codes, scale = PagedCache.to_code_layout(v)
    flat = codes.reshape(m, L, Hkv, P * D)
    t, e = torch.arange(P)[:, None], torch.arange(D)[None]
    at = (t & ~15) * D + e // 64 * 1024 + t // 4 % 4 * 256 + e % 16 * 16 + e // 16 % 4 * 4 + t % 4
    got = flat[1, 2, 1][at].view(torch.float8_e4m3fn).float() * scale[1, 2, 1].repeat_interleave(16)[:, None]
    back = PagedCache.from_code_layout(codes, scale)
    assert torch.equal(back[1, :, 2, 1], got)
    want = quantise_slots(v.float().view(m * P, L * Hkv, D)).view(m, P, L, Hkv, D)
    assert torch.equal(back, want.float())
    # at most half a step off: 2^-4 of the value, 2^-10 of the scale
    off = (back - v.float()).abs()
    assert bool((off <= 2.0 ** -4 * v.float().abs() * (1 + 2.0 ** -20) + 2.0 ** -10 * scale.max()).all())
    assert torch.equal(torch.sort(flat.flatten()).values, torch.sort(codes.flatten()).values)


def test_scales_of_unusual_blocks():
    v = torch.zeros((1, 64, 1, 1, D)).bfloat16()
    v[0, 20] = 3.0
    v[0, 33, 0, 0, 7] = math.inf
    v[0, 50, 0, 0, 7] = math.nan
    codes, scale = PagedCache.to_code_layout(v)
    s = scale[0, 0, 0]
    assert s[0] == 0 and s[1] == torch.tensor(3.0) / 448 and s[2].isnan() and s[3].isnan()
    assert torch.equal(PagedCache.from_code_layout(codes, scale)[0, :16].abs().max(), torch.tensor(0.0))


def test_quantise_takes_the_nearest_code():
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    table = table[table.isfinite()]
    x = torch.randn((1, 16, 1, D), generator=torch.Generator().manual_seed(2))
    back, scale = quantise(x)
    near = (x.double()[..., None] - scale.double()[:, None, :, None, None] * table).abs().amin(-1)
    assert bool(((back - x.double()).abs() <= near + 1e-9).all())


def test_visible_against_brute_force():
    live = np.array([1, 1, 0, 1, 1, 1, 0, 1], bool)
    for own in range(8):
        for window in (0, 1, 2, 3, 8, 20):
            for sinks in (0, 1, 3, 9):
                got = visible(live, own, window, sinks).numpy()
                want = [bool(live[j] and j <= own and (window == 0 or own - j < window or j < sinks)) for j in range(8)]
                assert got.tolist() == want


def test_attend_of_equal_keys_is_the_mean():
    k, v = torch.zeros((5, D)), torch.arange(5.0)[:, None].expand(5, D)
    out, lse, dev = attend(torch.ones((1, D)), k, v, torch.tensor([True, False, True, True, False]))
    assert torch.allclose(out, torch.full_like(out, 5 / 3)) and math.isclose(float(lse), math.log(3))
    assert torch.allclose(dev, torch.full_like(dev, (5 / 3 + 1 / 3 + 4 / 3) / 3))
    none = attend(torch.ones((1, D)), k, v, torch.zeros(5, dtype=torch.bool))
    assert torch.equal(none[0], torch.zeros(1, D).double()) and float(none[1]) == -math.inf


def test_forms_of_values():
    kw = dict(L=1, Hq=2, Hkv=1, d=D, P=16, S=1, max_pages=2, n_phys=2, device="cpu")
    assert PagedCache(**kw).v_pool is None and PagedCache(**kw).v_codes is None
    assert PagedCache(**kw, values=True).v_codes is None and PagedCache(**kw, values="e4m3").v_pool is None
    for bad in ("e5m2", 8, "yes"):
        with pytest.raises(ValueError):
            PagedCache(**kw, values=bad)
    c = PagedCache(**kw, values="e4m3")
    c.load_session(0, torch.randn(20, 1, 1, D), [0] * 20, [1, 0], budget=20, clock=20)
    v = torch.randn(20, 1, 1, D).bfloat16()
    c.load_values(0, v)
    back = PagedCache.from_code_layout(c.v_codes[[1, 0]], c.v_scale[[1, 0]]).flatten(0, 1)[:20]
    assert torch.equal(back, quantise_slots(v.float().flatten(1, 2)).view(20, 1, 1, D).float())
    assert torch.equal(c.v_open[0, 0, 0, :4], v[16:, 0, 0]) and not bool(c.v_open[0, 0, 0, 4:].any())
