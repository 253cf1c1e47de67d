"""The 256-row persistent products at MX4 weights, checked on their compiled code as the
128-row ones are (test_mx4_waits.py): the waits count operations issued after those they
wait for, so each stretch between two barriers holds at least as many as the count assumes,
and a tile's epilogue at least as many stores."""
import re

import pytest

from test_mx4_waits import asm  # noqa: F401  (the compiled code)

MOST = 63   # the counter's largest value: no wait at all


def _body(asm, act, epilogue):
    name = f"gemm_mx4_big_kernelILi{act}ELi{epilogue}ELi256E"
    start = next(i for i, l in enumerate(asm) if l.startswith("_Z") and name in l)
    end = next(i for i in range(start, len(asm)) if asm[i].startswith(".Lfunc_end"))
    return [l.split(";")[0].strip() for l in asm[start:end]]


def _stretches(body):
    """(matrix instructions, copies, scale loads, waits) between barriers, without what lies
    before the first and after the last."""
    mfma = copies = loads = 0
    waits, out = [], []
    for l in body:
        found = re.match(r"s_waitcnt .*?vmcnt\((\d+)\)", l)
        if found:
            waits.append(int(found[1]))
        elif l.startswith("buffer_load"):
            copies += l.endswith("lds")
            loads += not l.endswith("lds")
        mfma += l.startswith("v_mfma")
        if l == "s_barrier":
            out.append((mfma, copies, loads, waits))
            mfma = copies = loads = 0
            waits = []
    return out[1:]


def _stores(act, epilogue):
    """Of a tile's 128 rows of a wave, where no row's last scales are padded and no
    pre-activations are kept."""
    return 64 if epilogue else 8 if act == 0 else 32


@pytest.mark.parametrize("act,epilogue,more", [
    (0, 0, 4), (0, 1, 0), (0, 2, 0),    # (padded scales)
    (1, 0, 64), (1, 1, 0), (1, 2, 0)])  # (kept pre-activations)
def test_stores_are_as_many_as_the_waits_count(asm, act, epilogue, more):  # noqa: F811
    stores = sum(l.startswith("buffer_store") for l in _body(asm, act, epilogue))
    assert stores == _stores(act, epilogue) + more


@pytest.mark.parametrize("epilogue", [0, 1, 2])
def test_mx4_steps(asm, epilogue):  # noqa: F811
    """Two barriers a step: before the first lie the copies of A (a tile's first step: none,
    they were its predecessor's last) and six scales, before the second four copies of B,
    then the wait that leaves those 14 operations, in a tile's first step the stores as well
    (where the counter holds them).  The compiler's waits for scales come before it."""
    all_ = _stretches(_body(asm, 0, epilogue))
    assert len(all_) >= 8 and len(all_) % 2 == 0
    for i, ((m1, a, s1, _), (m2, b, s2, waits)) in enumerate(zip(all_[::2], all_[1::2])):
        assert m1 + m2 == (32 if i else 24)
        assert (a, s1) == ((4, 6) if i else (0, 6)) and (b, s2) == (4, 0)
        most = min(14 + (0 if i else _stores(0, epilogue)), MOST)
        assert most == MOST or waits[-1] <= most


@pytest.mark.parametrize("epilogue", [0, 1, 2])
def test_bf16_steps(asm, epilogue):  # noqa: F811
    """Four copies of activations, one of weights and two scales a step; the wait at its end
    leaves two steps' copies, in a tile's first two steps the stores as well."""
    all_ = _stretches(_body(asm, 1, epilogue))
    assert len(all_) >= 5
    for i, (m, copies, loads, waits) in enumerate(all_):
        assert m == (32 if i else 24) and copies == 5 and loads == 2
        early = 10 + (_stores(1, epilogue) if i < 2 else 0)
        assert early >= MOST or waits[-1] <= early
