"""The error bound that laep_block.h states for 8-bit checkpoints, over every exponent
that float32 has."""
import os
import re

import numpy as np
import pytest

import oracle.block as ob

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("exponent", range(-149, 128))
def test_error_bound(exponent):
    rng = np.random.default_rng(exponent + 200)
    v = rng.uniform(-1, 1, (64, 32))
    v[:, 5] = rng.choice([-1, 1], 64) * rng.uniform(1, 2, 64)       # the largest: exponent's
    v[0, 5], v[1, 5] = 1.0, 255 / 128
    with np.errstate(over="ignore", under="ignore"):
        v = np.ldexp(v, exponent).astype(np.float32).astype(np.float64)
    v[~np.isfinite(v)] = 0.0
    q, b = ob.act8_save(v)
    err = np.abs(ob.act8_load(q, b) - v).max(1)
    top = np.abs(v).max(1)
    step = np.ldexp(1.0, b[:, 0].astype(int) - 127)
    half = np.where(top > 127.5 * step, 1.0, 0.5) * step
    assert (err <= half).all()
    big = top >= 2.0 ** -120
    assert (top[big] >= 64 * step[big]).all() and (top[big] < 128 * step[big]).all()
    assert (half[big] <= np.where(top > 127.5 * step, 1 / 64, 1 / 128)[big] * top[big]).all()
    assert (b[~big] == 1).all() and (err[~big] <= 2.0 ** -127).all()


def test_the_bound_as_stated():
    """The documents say where 1/128 ends."""
    for path in ("include/laep_block.h", "paper_2601_14327_amd/csrc/act8.hip"):
        text = re.sub(r"\s*\n\s*(\*|//)?\s*", " ", open(os.path.join(ROOT, path)).read())
        assert "From 2^-120 up the largest magnitude takes 64 to 127 steps" in text, path
        assert "below 2^-120 steps are 2^-126 and the error at most 2^-127" in text, path
