"""tests/test_abi_paged_loop.py again, against the host code built with
AddressSanitizer and UndefinedBehaviorSanitizer (CPU only)."""
import os
import subprocess
import sys

import pytest

from paper_2506_12035_amd import build
from test_abi_sanitized import ROOT, _have_toolchain


@pytest.mark.skipif(not _have_toolchain(), reason="hipcc or clang's ASan runtime not installed")
def test_paged_loop_abi_under_address_and_undefined_behavior_sanitizers(tmp_path):
    lib = build.build_sanitized()
    env = dict(os.environ)
    env.update({
        "LD_PRELOAD": ":".join(p for p in (build.asan_runtime(), os.environ.get("LD_PRELOAD")) if p),
        "ASAN_OPTIONS": f"detect_leaks=0:alloc_dealloc_mismatch=0:verify_asan_link_order=0:"
                        f"halt_on_error=1:log_path={tmp_path / 'san'}",
        "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1",
        "MARCHE_LIB_PATH": lib,
    })
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_abi_paged_loop.py", "-q", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    reports = "".join(p.read_text() for p in tmp_path.glob("san*"))
    assert r.returncode == 0 and not reports, (r.stdout[-3000:] + r.stderr[-3000:] + reports[:4000])
    assert " passed" in r.stdout
