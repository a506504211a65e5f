"""The host side of causal attention and of the 4-bit cache (argument validation, sequence tables, the plans that calls are cut by)
under AddressSanitizer and UndefinedBehaviorSanitizer: csrc/causal_api.hip with stub launchers
(tests/host_sanitize/causal_driver.hip) that check every table and plan, over random calls.  CPU only: nothing is launched."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None and not os.path.exists(HIPCC), reason="hipcc not available")
def test_host_paths_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "host_sanitize_causal")
    csrc = os.path.join(ROOT, "paper_2503_12964_amd", "csrc")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Wno-unused-command-line-argument",
           "-Wno-inline-asm", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", csrc,
           os.path.join(csrc, "causal_api.hip"), os.path.join(ROOT, "tests", "host_sanitize", "causal_driver.hip"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    err = "\n".join(x for x in res.stderr.splitlines() if "is not a recognized feature for this target" not in x)
    assert res.returncode == 0, err[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert run.returncode == 0, (run.stdout[-2000:] + run.stderr[-4000:])
    assert run.stdout.strip().startswith("ok:"), run.stdout[-500:]
