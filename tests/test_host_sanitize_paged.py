"""The paged-cache entry points' host code built with AddressSanitizer and UndefinedBehaviorSanitizer (host code
only) and driven by tests/sanitize/paged_driver.cpp with calls that are refused, on the CPU."""

import os

import pytest

import test_host_sanitize as base
from paper_2606_10537_amd import build as B


@pytest.mark.skipif(not os.path.exists(base.HIPCC), reason="hipcc not installed")
def test_paged_validation_under_asan_ubsan():
    out_dir = os.path.join(base.PKG, "_build", "sanitize_paged")
    os.makedirs(out_dir, exist_ok=True)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    objs = []
    for src in ("pd_api.hip", "paged_api.hip"):
        o = os.path.join(out_dir, src.replace(".hip", ".o"))
        rc, out = base.run([B.HIPCC, *B.FLAGS, *san, "-c", os.path.join(B.CSRC, src), "-o", o])
        assert rc == 0, out[-3000:]
        objs.append(o)
    for src in B.SOURCES:   # the launchers, from the build or compiled here
        if src in ("pd_api.hip", "paged_api.hip"):
            continue
        o = os.path.join(B.BUILD, src.replace(".hip", ".o"))
        if not os.path.exists(o):
            o = os.path.join(out_dir, src.replace(".hip", ".o"))
            rc, out = base.run([B.HIPCC, *B.FLAGS, "-c", os.path.join(B.CSRC, src), "-o", o])
            assert rc == 0, out[-3000:]
        objs.append(o)
    drv = os.path.join(out_dir, "paged_driver.o")
    rc, out = base.run([B.HIPCC, "-x", "c++", "-std=c++17", "-O1", *san, f"-I{B.INCLUDE}", "-c",
                        os.path.join(base.ROOT, "tests", "sanitize", "paged_driver.cpp"), "-o", drv])
    assert rc == 0, out[-3000:]
    exe = os.path.join(out_dir, "paged_driver")
    rc, out = base.run([B.HIPCC, f"--offload-arch={B.ARCH}", *san, drv, *objs, "-o", exe])
    assert rc == 0, out[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", HIP_VISIBLE_DEVICES="")
    rc, out = base.run([exe], env=env, timeout=120)
    assert rc == 0 and "ok (0 failures)" in out, out[-4000:]
    assert "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
