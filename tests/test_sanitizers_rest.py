"""Sanitizer builds of the library's host code, on the CPU, for the entry points
that the drivers of tests/test_sanitizers.py do not call: AddressSanitizer and
UndefinedBehaviorSanitizer over their validation and size arithmetic
(tests/native/abi_sanitize_rest.cpp), ThreadSanitizer over eight host threads
(tests/native/abi_threads_rest.cpp).  The device code is built as usual and
never run; any report aborts the driver, which fails the test."""
import concurrent.futures
import glob
import os
import re
import subprocess

import pytest

from paper_2605_08755_amd import laq

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = "/opt/rocm/bin/hipcc"
CLANGXX = "/opt/rocm/lib/llvm/bin/clang++"


def run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-3000:] + r.stderr[-3000:]


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANGXX)), reason="needs the ROCm toolchain")
@pytest.mark.parametrize("driver,kinds,options,checks", [
    ("abi_sanitize_rest", "address,undefined", {"ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
                                               "UBSAN_OPTIONS": "print_stacktrace=1"}, 10000),
    ("abi_threads_rest", "thread", {"TSAN_OPTIONS": "halt_on_error=1:abort_on_error=1"}, 8 * 3000 * 2),
])
def test_validation_under_sanitizers(tmp_path, driver, kinds, options, checks):
    csrc = os.path.join(ROOT, "paper_2605_08755_amd", "csrc")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", csrc]
    host = []  # the host pass alone
    for flag in ["-fsanitize=" + k for k in kinds.split(",")] + ["-fno-sanitize-recover=all"]:
        host += ["-Xarch_host", flag]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops"] + host + inc + ["-c", src, "-o", obj])
        return obj
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, sorted(glob.glob(os.path.join(csrc, "*.hip")))))
    drv, exe = str(tmp_path / (driver + ".o")), str(tmp_path / driver)
    run([CLANGXX, "-std=c++17", "-O1", "-g", "-fsanitize=" + kinds, "-fno-sanitize-recover=all"] + inc +
        ["-c", os.path.join(HERE, "native", driver + ".cpp"), "-o", drv])
    run([HIPCC, "--offload-arch=gfx950"] + host + [drv] + objs + ["-o", exe, "-lpthread"])
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(os.environ, **options))
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-3000:] + r.stderr[-3000:]
    assert int(r.stdout.split()[1]) > checks


def test_every_entry_point_is_driven():
    """Each exported name stands in a driver of the host code's validation."""
    text = "".join(open(os.path.join(HERE, "native", d)).read() for d in ("abi_sanitize.cpp", "abi_sanitize_rest.cpp"))
    assert not [e for e in laq.EXPORTS if not re.search(r"\b" + e + r"\b", text)]
