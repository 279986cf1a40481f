"""Host code of the operators around the layer under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, no GPU code is instrumented): the stored
form and the quantiser of four-bit weights, and the entry points' argument checks and choices of kernels."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_16795_amd", "csrc")
UNITS = ["qmoe_int4_host.cpp", "qmoe_host.cpp", "qmoe_api.hip", "qmoe_norm.hip", "qmoe_route.hip", "qmoe_int4.hip"]
HOST_ONLY = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]


def test_operators_host_side_under_asan_and_ubsan(tmp_path):
    from paper_2310_16795_amd import build as B

    runtimes = [os.path.join(base, f) for base, _, files in os.walk("/opt/rocm/lib/llvm/lib/clang") for f in files if f == "libclang_rt.asan-x86_64.so"]
    if not runtimes:
        pytest.skip("clang's shared ASan runtime is not installed")
    B.build_library(incremental=True)  # the objects that the sanitized ones are linked with
    flags = ["-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    objects, jobs = [], []
    for u in UNITS:
        objects.append(str(tmp_path / (os.path.splitext(u)[0] + ".o")))
        jobs.append(subprocess.Popen(["hipcc", *flags, *HOST_ONLY, "-c", os.path.join(CSRC, u), "-o", objects[-1]], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for j in jobs:
        out = j.communicate()[0]
        assert j.returncode == 0, out[-3000:]
    others = [os.path.join(B.OBJ, os.path.splitext(u)[0] + ".o") for u in B.UNITS if u not in UNITS]
    lib = str(tmp_path / "libqmoe_san.so")
    subprocess.check_call(["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", *HOST_ONLY[:4], "-shared-libsan", "-o", lib, *objects, *others])
    names = subprocess.check_output(["nm", objects[0]], text=True)
    assert "__asan_report" in names and "__ubsan_handle" in names  # instrumented
    env = {**os.environ, "QMOE_LIBRARY": lib, "LD_PRELOAD": " ".join(x for x in (os.environ.get("LD_PRELOAD"), runtimes[0]) if x),
           "ASAN_OPTIONS": "detect_leaks=0:verify_asan_link_order=0:abort_on_error=0:exitcode=23",
           "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1:exitcode=23"}
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "not gpu", "-p", "no:cacheprovider", "tests/test_operators_host.py"], cwd=ROOT, env=env,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-4000:]
