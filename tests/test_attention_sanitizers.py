"""Host side of attention (attention_plan.cpp), compiled with AddressSanitizer and UndefinedBehaviorSanitizer and driven by
tests/sanitize_attention.cpp over random and extreme batches."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import ROOT, SAN


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans_of_attention_under_address_and_undefined_behaviour_sanitizers(tmp_path):
    exe = str(tmp_path / "sanitize_attention")
    sources = [os.path.join(ROOT, "paper_2411_00915_amd", "csrc", "attention_plan.cpp"), os.path.join(ROOT, "tests", "sanitize_attention.cpp")]
    subprocess.run(["g++", "-o", exe, "-std=c++17", "-Wall"] + SAN + sources + ["-static-libasan", "-static-libubsan"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0 and "sanitize_attention: ok" in res.stdout, f"{res.stdout[-2000:]}\n{res.stderr[-6000:]}"
    assert "runtime error" not in res.stderr and "ERROR: AddressSanitizer" not in res.stderr and "LeakSanitizer" not in res.stderr, res.stderr[-6000:]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_that_share_memory_are_found(tmp_path):
    exe = str(tmp_path / "sanitize_memory_rows")
    sources = [os.path.join(ROOT, "paper_2411_00915_amd", "csrc", "attention_plan.cpp"), os.path.join(ROOT, "tests", "sanitize_memory_rows.cpp")]
    subprocess.run(["g++", "-o", exe, "-std=c++17", "-Wall"] + SAN + sources + ["-static-libasan", "-static-libubsan"], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "sanitize_memory_rows: ok" in res.stdout, f"{res.stdout[-2000:]}\n{res.stderr[-6000:]}"
    assert "runtime error" not in res.stderr, res.stderr[-6000:]
