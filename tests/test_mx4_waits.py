"""The 128-row persistent products at MX4 weights, checked on their compiled code: between
two barriers of a k-loop lie the copies into LDS that the wait counts assume, and no other
load, whose arrival would be waited for, and all older copies with it."""
import re
import subprocess

import pytest

from paper_2601_14327_amd import build


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "gemm_mx4_big.s"
    subprocess.run([build._hipcc(), "-x", "hip", *build.COMMON, *build.HIP_FLAGS,
                    "--cuda-device-only", "-S", f"{build.CSRC}/gemm_mx4_big.hip", "-o", str(out)],
                   check=True, stderr=subprocess.DEVNULL, timeout=300)
    return out.read_text().splitlines()


def _steps(asm, name):
    """(matrix instructions, copies, other loads, last wait) between barriers, where a wave
    has both of its 32-row blocks."""
    start = next(i for i, l in enumerate(asm) if l.startswith("_Z") and name in l)
    end = next(i for i in range(start, len(asm)) if asm[i].startswith(".Lfunc_end"))
    mfma = copies = loads = 0
    wait, out = None, []
    for l in (l.split(";")[0].strip() for l in asm[start:end]):
        found = re.match(r"s_waitcnt .*?vmcnt\((\d+)\)", l)
        if found:
            wait = int(found[1])
        elif re.match(r"(buffer|global|flat|scratch)_load", l):
            copies += l.endswith("lds")
            loads += not l.endswith("lds")
        mfma += l.startswith("v_mfma")
        if l == "s_barrier":
            out.append((mfma, copies, loads, wait))
            mfma = copies = loads = 0
            wait = None
    return [s for s in out if s[0] == 16]


@pytest.mark.parametrize("act,epilogue,stores", [
    (0, 0, 6), (0, 1, 32), (0, 2, 32),    # (4, and 2 where a row's last scales are padded)
    (1, 0, 48), (1, 1, 32), (1, 2, 32)])  # (16, and 32 of kept pre-activations)
def test_stores_are_as_many_as_the_waits_count(asm, act, epilogue, stores):
    """A tile's first waits leave its predecessor's stores in flight: none is merged."""
    name = f"gemm_mx4_big_kernelILi{act}ELi{epilogue}ELi128E"
    start = next(i for i, l in enumerate(asm) if l.startswith("_Z") and name in l)
    end = next(i for i in range(start, len(asm)) if asm[i].startswith(".Lfunc_end"))
    assert sum(l.strip().startswith("buffer_store") for l in asm[start:end]) == stores


@pytest.mark.parametrize("epilogue,stores", [(0, 16), (1, 32), (2, 32)])
def test_bf16_steps(asm, epilogue, stores):
    """Two copies of activations and one of weights a step, in two of four steps scales as
    well; the wait leaves those of three steps, less the last one's weights."""
    steps = _steps(asm, f"gemm_mx4_big_kernelILi1ELi{epilogue}ELi128E")
    assert len(steps) >= 8 and not [s for s in steps if s[2]]
    assert {s[1] for s in steps} == {3, 4} and {s[3] for s in steps} <= {11, 11 + stores}


@pytest.mark.parametrize("epilogue,stores", [(0, 4), (1, 32), (2, 32)])
def test_mx4_steps(asm, epilogue, stores):
    """Two copies of activations, four of weights and two of scales a step; the wait leaves
    one step's."""
    steps = _steps(asm, f"gemm_mx4_big_kernelILi0ELi{epilogue}ELi128E")
    assert steps and not [s for s in steps if s[2]]
    assert {s[1] for s in steps} == {8} and {s[3] for s in steps} <= {8, 8 + stores}
