"""The CPU tests of the adapters and tensor lists again, against the host-sanitizer build of the C-ABI layer."""
import os
import subprocess
import sys

import pytest

from test_abi_sanitized import ROOT, _build_module


def test_adapters_and_lists_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    b = _build_module()
    try:
        lib, rt = b.build_host_sanitized(str(tmp_path)), b.asan_runtime()
    except FileNotFoundError as e:
        pytest.skip(str(e))
    env = dict(os.environ, GM_LIBRARY_PATH=lib, LD_PRELOAD=rt,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_lora_cpu.py"), "-q", "-x",
                        "-p", "no:cacheprovider"], env=env, capture_output=True, text=True, timeout=600, cwd=ROOT)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0 and "Sanitizer" not in out and " passed" in r.stdout, out
