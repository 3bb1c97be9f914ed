"""Properties of the generated gfx950 code that the 8-bit float products rely on (no GPU).

The largest tiles keep their 256 sums a lane in accumulator registers, through matrix instructions written as inline
assembly, whose hazards the compiler does not know.  The kernel is right only while nothing else in its loop touches
those registers (no move, no spill), each such instruction comes behind two wait states, and nothing reads the sums
between the loop's end and the settling wait."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2405_03594_amd import build as B

SRC = os.path.join(B.CSRC, "k_fp8_gemm.hip")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(B.HIPCC) and not shutil.which("hipcc"):
        pytest.skip("hipcc is not available")
    out = tmp_path_factory.mktemp("asm") / "k_fp8_gemm.s"
    r = subprocess.run([B.HIPCC, *[f for f in B.CFLAGS if f != "-fPIC"], "-S", "--cuda-device-only", SRC, "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    text, found = out.read_text(), {}
    for m in re.finditer(r"^(_Z\w*(?:k_fp8_tile|k_fp8_mixed)\w*):", text, re.M):
        body = text[m.start():text.index(".Lfunc_end", m.start())]
        # a line of inline assembly is marked, other comments are left out
        lines, ours = [], False
        for l in body.split("\n"):
            if "#ASMSTART" in l or "#ASMEND" in l:
                ours = "#ASMSTART" in l
            else:
                l = l.split(";")[0].strip()
                lines.append("asm " + l if l and ours else l)
        found[m.group(1)] = [l for l in lines if l]
    assert found
    return found


def _accumulating(lines):
    return [i for i, l in enumerate(lines) if l.startswith("asm v_mfma_scale_f32_16x16x128_f8f6f4")]


def test_sums_stay_in_accumulator_registers(kernels):
    large = {n: l for n, l in kernels.items() if _accumulating(l)}
    assert len(large) >= 4                              # uniform and mixed launches, two types
    for name, lines in large.items():
        at = _accumulating(lines)
        assert len(at) == 64, name                      # a stage's
        for i in at:
            assert lines[i - 1] == "asm s_nop 1", (name, lines[i - 1])
            m = re.match(r"asm v_mfma\S+ (a\[\d+:\d+\]), v\[\S+\], v\[\S+\], (a\[\d+:\d+\]), v\d+, v\d+", lines[i])
            assert m and m.group(1) == m.group(2), (name, lines[i])
        loop = lines[at[0]:at[-1] + 1]
        for l in loop:
            assert not l.startswith(("v_accvgpr", "scratch_")), (name, l)
            if not l.startswith("asm v_mfma"):
                assert not re.search(r"\ba(\d+|\[\d+:\d+\])", l), (name, l)
        # behind the loop: 48 wait states before the first read of a sum
        rest = lines[at[-1] + 1:]
        settle = next(i for i in range(len(rest)) if rest[i:i + 3] == ["asm s_nop 15"] * 3)
        assert not any(re.search(r"\ba(\d+|\[\d+:\d+\])", l) for l in rest[:settle]), name


def test_waits_are_counted(kernels):
    """In a loop's stage the only wait for requests is the counted one in front of the barrier: deeper rings keep theirs."""
    seen = 0
    for name, lines in kernels.items():
        m = re.search(r"k_fp8_tileINS_\w+?ELb[01]ELi\dELi\dELi\dELi\dELi(\d)E", name)
        if not m or int(m.group(1)) == 2:
            continue
        seen += 1
        barriers = [i for i, l in enumerate(lines) if l == "s_barrier"]
        inside = next(i for i in barriers[1:] if any("v_mfma" in l for l in lines[i:i + 60]))
        start = max(i for i, l in enumerate(lines[:inside]) if l.startswith(".LBB"))
        end = next(i for i in range(inside, len(lines)) if lines[i].startswith("s_cbranch"))
        waits = [l for l in lines[start:end] if l.startswith("s_waitcnt") and "vmcnt" in l]
        assert len(waits) == 1 and "vmcnt(0)" not in waits[0], (name, waits)
    assert seen >= 4
