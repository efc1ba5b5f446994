"""The attention operators' host code (buckets, argument checks, plans, workspace sizes)
under AddressSanitizer and UndefinedBehaviorSanitizer, as test_sanitized_host.py does for
the stage and the allocator (CPU only; the child is tests/_sanitized_attn_driver.py)."""
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.timeout(900)
def test_attention_host_paths_under_sanitizers():
    from paper_2202_11836_amd import build as B
    try:
        lib = B.build_sanitized()
        rt = B.sanitizer_runtime()
    except (RuntimeError, OSError) as e:  # no hipcc / sanitizer runtime here
        pytest.skip(str(e))
    env = dict(os.environ, LD_PRELOAD=rt, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, os.path.join(HERE, "_sanitized_attn_driver.py"), lib], env=env,
                       capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "sanitized attention host paths: ok" in r.stdout
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
