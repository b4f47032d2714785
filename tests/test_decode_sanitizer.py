"""The decode operators' checks of their arguments under AddressSanitizer and
UndefinedBehaviorSanitizer: tests/decode_args.cpp compiles the library's host
layer in, fills a handle by hand and replaces the launchers, so that every
refusal is reached with a handle and without a GPU.  (tests/abi_sanitize.c
covers the other entry points, on the built library and without a handle.)"""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_arguments_of_the_decode_operators_under_sanitizers(tmp_path):
    exe = tmp_path / "decode_args"
    # (what the checks do not reach, the launchers of the step and the HIP runtime, stays unresolved)
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "decode_args.cpp"),
           "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "passed under the sanitizers" in r.stdout
