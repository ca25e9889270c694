"""The validation of the embedding, the layer norm, the cross-entropy loss and gradient clipping under AddressSanitizer
and UndefinedBehaviorSanitizer, on the host-only build of test_sanitized_host.py."""
import os
import subprocess
import sys

from test_sanitized_host import ROOT, sanitized_builds  # noqa: F401

MODULES = ["tests/test_abi_host_language.py"]


def test_language_validation_clean_under_address_and_ub_sanitizers(sanitized_builds):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=sanitized_builds["runtime"], MT_LIB_OVERRIDE=sanitized_builds["lib"],
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:alloc_dealloc_mismatch=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu", "-p", "no:cacheprovider", *MODULES],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    text = r.stdout + r.stderr
    assert "AddressSanitizer" not in text and "runtime error:" not in text, text[-6000:]
    assert r.returncode == 0, text[-6000:]
    assert " passed" in r.stdout
