"""The paged cache's host side (argument checks, plans, workspace sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer, without recovery: the library
sources (only their host code is instrumented, nothing is launched) and
tests/sanitize/paged_driver.cpp.  The build is cached per source digest in the
system temp directory."""
import os
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_sanitizers import CSRC, ENV, HIPCC, ROOT, SAN, _digest, _run

SOURCES = ["api", "topk", "ngram", "round", "tree_build", "tree_attn", "accept", "api_paged", "pages", "paged_attn"]


def test_paged_host_under_asan_ubsan():
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    srcs = [os.path.join(CSRC, f + ".hip") for f in SOURCES]
    driver = os.path.join(SAN, "paged_driver.cpp")
    hdrs = [os.path.join(CSRC, "common.hpp"), os.path.join(CSRC, "paged.hpp"),
            os.path.join(ROOT, "include", "presto.h"), driver]
    build = os.path.join(tempfile.gettempdir(), f"presto_san_paged_{_digest(srcs + hdrs)}")
    exe = os.path.join(build, "paged_driver")
    if not os.path.exists(exe):
        os.makedirs(build, exist_ok=True)
        inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
        san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
               "-Xarch_host", "-fno-sanitize-recover=all"]

        def compile_one(name):
            obj = os.path.join(build, name + ".o")
            _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
                  "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *san, *inc,
                  "-c", os.path.join(CSRC, name + ".hip"), "-o", obj])
            return obj

        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as ex:
            objs = list(ex.map(compile_one, SOURCES))
        drv = os.path.join(build, "driver.o")
        _run([HIPCC, "-O1", "-g", "-std=c++17", *san, *inc, "-c", driver, "-o", drv])
        _run([HIPCC, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined",
              "-fno-gpu-sanitize", drv, *objs, "-o", exe + ".tmp"])
        os.replace(exe + ".tmp", exe)
    r = _run([exe], env=dict(ENV, ASAN_OPTIONS="detect_leaks=0"), timeout=300)
    assert "paged driver: ok" in r.stdout
