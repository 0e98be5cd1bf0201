"""The host side of the sampling and clipping calls under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only):
their HIP sources with the sanitizers on the host pass, driven by tests/sanitize/operator_args.c."""
import os

import pytest

from tests.test_sanitizers import CLANG, HERE, HIPCC, HOST_SAN, ROCM, ROOT, _run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="ROCm compilers not available")
def test_operator_host_checks_under_asan_ubsan(tmp_path):
    csrc = os.path.join(ROOT, "paper_2606_05597_amd", "csrc")
    flags = ["--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"), "-I" + csrc, *HOST_SAN]
    objs = []
    for f in ("sampling.hip", "clip.hip"):
        objs.append(str(tmp_path / (f + ".o")))
        _run([HIPCC, *flags, "-c", os.path.join(csrc, f), "-o", objs[-1]])
    lib = str(tmp_path / "liboperators_san.so")
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *HOST_SAN, *objs, "-o", lib])
    exe = str(tmp_path / "operator_args")
    _run([CLANG, "-std=c11", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROOT, "include"),
          "-I" + os.path.join(ROCM, "include"), "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
          os.path.join(HERE, "operator_args.c"), lib, "-Wl,-rpath," + str(tmp_path), "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    assert "operator argument checks ok" in _run([exe], env=env).stdout
