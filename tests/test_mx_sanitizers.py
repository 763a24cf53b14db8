"""The microscaled C entry points, built host-only with mock launchers, under AddressSanitizer and
UndefinedBehaviorSanitizer: argument checks, chunks of tokens, offsets and workspace sizes."""
import os

import pytest

from tests.test_sanitizers import CLANG, HERE, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(CLANG), reason="ROCm clang not installed")
def test_mx_abi_under_sanitizers_with_mock_launchers(tmp_path):
    exe = str(tmp_path / "mx_mock")
    csrc = os.path.join(ROOT, "paper_2312_06881_amd", "csrc")
    _run([CLANG, "-x", "hip", "--offload-host-only", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc,
          os.path.join(csrc, "dyad_abi.hip"), os.path.join(csrc, "mx_abi.hip"), os.path.join(HERE, "mx_mock.cpp"),
          "-o", exe, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    r = _run([exe], env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
    assert "mx mock ok" in r.stdout
