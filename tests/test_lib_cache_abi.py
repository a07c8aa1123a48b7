"""The paged cache's entry points from plain C, and under sanitizers (CPU).

``tests/c_abi/host_cache.c`` includes only ``include/bsr.h`` and drives a
host-only context.  It is linked against libbsr.so, and then against the host
code built with AddressSanitizer and UndefinedBehaviorSanitizer (host code only;
the kernels of the attention are left out, since no call gets that far).
"""

import os
import shutil
import subprocess

import pytest

from paper_2608_17826_amd import bsr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "c_abi", "host_cache.c")
CSRC = os.path.join(ROOT, "paper_2608_17826_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# host code only: each sanitizer flag applies to the host pass
SANITIZE = "-Xarch_host -fsanitize=address -Xarch_host -fsanitize=undefined -Xarch_host -fno-omit-frame-pointer".split()


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_plain_c_consumer(tmp_path):
    exe = str(tmp_path / "host_cache")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", f"-I{ROOT}/include", SRC,
                    f"-L{os.path.dirname(bsr.LIB_PATH)}", "-lbsr",
                    f"-Wl,-rpath,{os.path.dirname(bsr.LIB_PATH)}", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stderr


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_host_code_clean_under_asan_and_ubsan(tmp_path):
    common = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", f"-I{ROOT}/include", f"-I{CSRC}",
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    stub = tmp_path / "launch_attention.cpp"
    stub.write_text('#include "bsr_cache.h"\nnamespace bsr {\n'
                    "hipError_t launch_attention(const AttnParams&, hipStream_t) { return hipErrorUnknown; }\n}\n")
    objs = []
    for src, lang in (("bsr_runtime.cpp", []), ("bsr_file_tier.cpp", []), ("bsr_kernels.hip", ["-x", "hip"]),
                      ("bsr_cache.cpp", []), ("bsr_cache.hip", ["-x", "hip"]), (str(stub), [])):
        o = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run([HIPCC, *common, *SANITIZE, *lang, "-c", os.path.join(CSRC, src), "-o", o],
                       check=True, capture_output=True)
        objs.append(o)
    drv = str(tmp_path / "drv.o")
    subprocess.run([HIPCC, "-std=c11", "-x", "c", "-g", f"-I{ROOT}/include", *SANITIZE, "-c", SRC, "-o", drv],
                   check=True, capture_output=True)
    exe = str(tmp_path / "host_cache_asan")
    subprocess.run([HIPCC, "--offload-arch=gfx950", *SANITIZE, drv, *objs, "-o", exe, "-lpthread"],
                   check=True, capture_output=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stderr[-4000:]
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    assert r.stdout == "ok\n"
