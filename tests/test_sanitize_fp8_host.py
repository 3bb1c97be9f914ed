"""Code of the 8-bit float linears and of AdamW under sanitizers on the CPU: the functions that the streaming kernel takes
its blocks and their scale bytes by, compiled for the host, and the host checks of every entry point."""
import concurrent.futures as cf
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


@pytest.mark.timeout(600)
def test_host_checks(tmp_path):
    """Every entry point of the 8-bit floats and of AdamW with sizes and arguments at their limits, its host code under
    AddressSanitizer and UndefinedBehaviorSanitizer."""
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    san = [a for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for a in ("-Xarch_host", f)]
    csrc = os.path.join(ROOT, "paper_2405_03594_amd", "csrc")
    names = ["spl_fp8.hip", "k_fp8_gemm.hip", "k_fp8_stream.hip", "k_fp8_quant.hip", "k_adamw.hip"]
    sources = [os.path.join(csrc, n) for n in names] + [os.path.join(ROOT, "tests", "sanitize", "fp8_host_checks.cpp")]

    def compile_one(src):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", *san, *INC, "-Xclang", "-target-feature",
              "-Xclang", "-packed-fp32-ops", "-c", src, "-o", obj], str(tmp_path))
        return obj

    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, sources))
    exe = str(tmp_path / "checks")
    _run([HIPCC, "--offload-arch=gfx950", *san, *objs, "-o", exe], str(tmp_path))
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")
    r = subprocess.run([exe], cwd=str(tmp_path), capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout[-2000:] + r.stderr[-3000:]
