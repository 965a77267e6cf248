"""The host side of pwlq_attention.h under AddressSanitizer and UndefinedBehaviorSanitizer, as test_abi_sanitized has it for the rest."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_side_of_attention_passes_under_asan_and_ubsan():
    from paper_2002_00104_amd import build
    runtime = build.sanitizer_runtime()
    if not runtime:
        pytest.skip("the compiler has no shared AddressSanitizer runtime")
    env = dict(os.environ, PWLQ_LIB=build.build_sanitized(), ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    env["LD_PRELOAD"] = runtime + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "tests/test_attention_abi_cpu.py",
                        "tests/test_attention_abi_ends_cpu.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = (r.stdout + r.stderr)[-3000:]
    assert r.returncode == 0, tail
    assert " passed" in r.stdout and "failed" not in r.stdout, tail
    assert "Sanitizer" not in r.stderr and "runtime error" not in r.stderr, tail
