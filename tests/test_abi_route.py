"""Host-side checks of the choices' and the mixture's entry points: struct layouts against the
binding, and the host code of every source under AddressSanitizer and
UndefinedBehaviorSanitizer on the CPU, driven by tests/asan/route_driver.cpp against the
stand-in HIP runtime of tests/asan/hip_stub.cpp."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_2407_00051_amd as sg
from paper_2407_00051_amd.build import SOURCES
from tests.test_abi_sanitized import ASAN, CLANG, CSRC, HIPCC, ROOT, SAN, _run


def test_struct_layout_matches_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc unavailable")
    structs = {"sagips_choices": sg.Choices, "sagips_choice_grads": sg.ChoiceGrads, "sagips_routed": sg.Routed}
    lines = []
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("=MAX_TOP %d\\n", SAGIPS_MAX_TOP);')
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "sagips.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    for line in subprocess.check_output([str(exe)], text=True).splitlines():
        key, value = line.split()
        if key.startswith("="):
            assert getattr(sg, key[1:]) == int(value), key
        elif "." in key:
            name, field = key.split(".")
            assert getattr(structs[name], field).offset == int(value), key
        else:
            assert ctypes.sizeof(structs[key]) == int(value), key


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="hipcc / clang++ unavailable")
def test_route_host_code_under_sanitizers(tmp_path):
    objs = []
    for s in SOURCES:
        o = str(tmp_path / (s + ".o"))
        _run([HIPCC, "--cuda-host-only", "-x", "hip", "-std=c++17", "-O1", "-g", "-fPIC", *SAN,
              "-c", os.path.join(CSRC, s), "-o", o])
        objs.append(o)
    undef = _run(["nm", "-u", *objs]).stdout
    fat = sorted(set(re.findall(r"\b(__hip_fatbin_[0-9a-f]+)\b", undef)))
    fat_src = tmp_path / "fatbins.cpp"
    fat_src.write_text("".join(f'extern "C" const unsigned char {n}[16] = {{0}};\n' for n in fat))
    flags = ["-std=c++17", "-O1", "-g", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
             "-I" + os.path.join(ROOT, "include"), "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-fno-omit-frame-pointer"]
    extra = []
    for src in (os.path.join(ASAN, "hip_stub.cpp"), os.path.join(ASAN, "route_driver.cpp"), str(fat_src)):
        o = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([CLANG, *flags, "-c", src, "-o", o])
        extra.append(o)
    exe = str(tmp_path / "route_driver")
    _run([CLANG, "-fsanitize=address,undefined", *objs, *extra, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:allocator_may_return_null=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout[-3000:])
    assert r.returncode == 0, f"driver failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    assert "ALL OK" in r.stdout
