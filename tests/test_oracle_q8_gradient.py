"""How far the input gradient of a layer of 8-bit rows is from that of the unrounded gradient rows.

Each value of dy w_scale is off by half a step of its row at most, so its square by (step / 2)^2. The errors of
a row meet the weight's columns, whole numbers of random signs, in a sum whose mean square is that of the errors
times the weight's: the norm over many columns stays below sqrt(sum (step / 2)^2 w^2), up to the spread of such
a norm over 256 columns (1 / sqrt(512) of it, four times that allowed). A bound for every single column would be
sqrt(n) times as wide."""

import numpy as np
import pytest

from oracle import q8


@pytest.mark.parametrize("kind", ["normal", "heavy", "loud"])
@pytest.mark.parametrize("n", [768, 4096, 11008])
def test_input_gradient_near_that_of_unrounded_rows(n, kind):
    rng = np.random.default_rng(n)
    k, m = 256, 32
    w = rng.standard_normal((n, k)) * 0.02 * np.exp(0.5 * rng.standard_normal((n, 1)))
    scale = (np.abs(w).max(1) / 127.0).astype(np.float32).astype(np.float64)
    w = np.clip(np.rint(w / scale[:, None]), -127, 127)
    dy = (rng.standard_t(3, (m, n)) if kind == "heavy" else rng.standard_normal((m, n))) * 1e-3
    if kind == "loud":
        dy[:, :: n // 3] *= 20.0
    t = dy * scale
    real, got = t @ w, q8.linear_bwd(dy, w, scale)
    off = np.linalg.norm(got - real, axis=1)
    step = np.abs(t).max(axis=1) / 127.0
    bound = step / 2.0 * np.sqrt((w * w).sum())
    assert (off <= (1.0 + 4.0 / np.sqrt(2.0 * k)) * bound).all()
