"""The host side of the trees' and the pages' operators under AddressSanitizer, as
test_sanitizers_paged.py does for the others of a paged step."""
import os
import subprocess
import sys

import pytest

from test_sanitizers import ROOT, B, _asan_runtime


def test_passes():
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("clang's AddressSanitizer runtime is not installed")
    lib = B.build_asan()
    for src in ("tree.hip", "pages.hip"):
        obj = os.path.join(B.ASAN_DIR, src + ".o")
        assert os.path.exists(obj) and b"__asan_report" in open(obj, "rb").read(), src
    env = dict(os.environ, LD_PRELOAD=rt, PLORA_LIB=lib,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                          "-m", "not gpu", os.path.join(ROOT, "tests", "test_tree_abi.py"),
                          os.path.join(ROOT, "tests", "test_pages_abi.py")],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = res.stdout + res.stderr
    assert "AddressSanitizer" not in out, out[-4000:]
    assert res.returncode == 0 and " passed" in res.stdout, out[-4000:]
