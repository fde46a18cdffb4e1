"""Ends of the ranges that the learning entry points accept: their host code under the sanitizers on
the CPU, driven by tests/asan/learn_edges_driver.cpp against the stand-in HIP runtime of
tests/asan/hip_stub.cpp."""
import os
import re
import subprocess

import pytest

from paper_2407_00051_amd.build import SOURCES
from tests.test_abi_sanitized import ASAN, CLANG, CSRC, HIPCC, ROOT, SAN, _run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="hipcc / clang++ unavailable")
def test_edges_of_the_learning_calls(tmp_path):
    procs, objs = [], []
    for s in SOURCES:
        objs.append(str(tmp_path / (s + ".o")))
        procs.append(subprocess.Popen([HIPCC, "--cuda-host-only", "-x", "hip", "-std=c++17", "-O1", "-g", "-fPIC", *SAN,
                                       "-c", os.path.join(CSRC, s), "-o", objs[-1]], stdout=subprocess.DEVNULL, stderr=subprocess.PIPE))
    for s, p in zip(SOURCES, procs):
        err = p.communicate()[1].decode()
        assert p.returncode == 0, f"{s}:\n{err[-4000:]}"
    undef = _run(["nm", "-u", *objs]).stdout
    fat = sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", undef)))
    fat_src = tmp_path / "fatbins.cpp"
    fat_src.write_text("".join(f'extern "C" const unsigned char {n}[16] = {{0}};\n' for n in fat))
    flags = ["-std=c++17", "-O1", "-g", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
             "-I" + os.path.join(ROOT, "include"), "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-fno-omit-frame-pointer"]
    extra = []
    for src in (os.path.join(ASAN, "hip_stub.cpp"), os.path.join(ASAN, "learn_edges_driver.cpp"), str(fat_src)):
        extra.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([CLANG, *flags, "-c", src, "-o", extra[-1]])
    exe = str(tmp_path / "driver")
    _run([CLANG, "-fsanitize=address,undefined", *objs, *extra, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:allocator_may_return_null=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "ALL OK" in r.stdout, f"driver failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
