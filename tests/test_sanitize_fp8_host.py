"""Code of the 8-bit float linears under UndefinedBehaviorSanitizer on the CPU: the functions that the streaming kernel takes
its blocks and their scale bytes by, compiled for the host."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
HOST_SAN = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all"]
INC = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2405_03594_amd", "csrc")]


def _run(cmd, cwd, timeout=300):
    r = subprocess.run(cmd, cwd=cwd, capture_output=True, text=True, timeout=timeout)
    assert r.returncode == 0, f"{' '.join(cmd[:3])} ... failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
    return r.stdout


def test_stream_runs(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "runs")
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", *HOST_SAN, *INC, "-Xclang", "-target-feature", "-Xclang",
          "-packed-fp32-ops", os.path.join(ROOT, "tests", "sanitize", "fp8_stream_runs.hip"), "-o", exe], str(tmp_path))
    assert _run([exe], str(tmp_path)).startswith("ok ")
