"""The host side of the paged operators under AddressSanitizer: test_paged_abi.py
against the library whose entry points' files are instrumented, as
test_sanitizers.py does for the others."""
import os
import re
import subprocess
import sys

import pytest

from test_sanitizers import ROOT, B, _asan_runtime


def test_every_file_with_entry_points_is_instrumented_and_passes():
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("clang's AddressSanitizer runtime is not installed")
    lib = B.build_asan()
    names = []
    for src in B.SRCS:
        if re.search(r'^extern "C"', open(src).read(), re.M):
            names.append(os.path.basename(src))
            obj = os.path.join(B.ASAN_DIR, names[-1] + ".o")
            assert os.path.exists(obj) and b"__asan_report" in open(obj, "rb").read(), names[-1]
    assert {"plora.hip", "attn_plan.hip", "attn_paged.hip", "kv_plan.hip", "rope.hip"} <= set(names)
    env = dict(os.environ, LD_PRELOAD=rt, PLORA_LIB=lib,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                          "-m", "not gpu", os.path.join(ROOT, "tests", "test_paged_abi.py")],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = res.stdout + res.stderr
    assert "AddressSanitizer" not in out, out[-4000:]
    assert res.returncode == 0, out[-4000:]
    assert " passed" in res.stdout
