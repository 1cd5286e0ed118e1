"""The dense layers' host code (argument checks, planning, workspace sizes)
compiled for the host only with AddressSanitizer and
UndefinedBehaviorSanitizer, driven by tests/sanitize/dense_driver.c (CPU only).

Host-only objects refer to their device code objects by symbol; empty
stand-ins are linked in, and no call of the driver reaches a kernel.
"""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1512_06473_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
HIPCC, CLANG = os.path.join(ROCM, "bin", "hipcc"), os.path.join(ROCM, "llvm", "bin", "clang")
HOST_SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
            "-fno-sanitize-recover=all"]
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g", "-O1"]
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".hip", ".cpp")))


def run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300, **kw)
    assert r.returncode == 0, (cmd[-1], r.stdout[-500:] + r.stderr[-3000:])
    return r.stdout


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_dense_host_code_under_sanitizers(tmp_path):
    def compile_host(src):
        # the dense sources and the workspace with sanitizers, what they only link with without
        san = HOST_SAN if src.startswith("dense_") or src == "scratch.cpp" else []
        obj = str(tmp_path / (os.path.splitext(src)[0] + ".o"))
        run([HIPCC, "-x", "hip", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-fPIC", "-std=c++17"] + san +
            ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, src), "-o", obj])
        return obj

    with cf.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_host, SOURCES))
    undef = set()
    for o in objs:
        undef.update(re.findall(r"\b(__hip_fatbin_\w+)", run(["nm", "-u", o])))
    stub = tmp_path / "stubs.c"
    stub.write_text("".join("__attribute__((aligned(4096))) const char %s[4096] = {0};\n" % s for s in sorted(undef)))
    driver, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    run([CLANG] + SAN + ["-I", os.path.join(ROOT, "include"), "-c",
                         os.path.join(ROOT, "tests", "sanitize", "dense_driver.c"), "-o", driver])
    run([CLANG, "-c", str(stub), "-o", str(tmp_path / "stubs.o")])
    run([CLANG + "++"] + SAN + ["-o", exe, driver] + objs + [str(tmp_path / "stubs.o"), "-L", os.path.join(ROCM, "lib"),
                                                             "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib")])
    # The HIP runtime keeps allocations until exit: leak detection off here.
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    out = run([exe], env=env)
    assert out.strip().endswith("ok"), out
    print(out)
