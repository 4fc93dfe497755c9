"""How far an element of a checkpoint may move, as dcp.h states it, on the definition's own
oracle: random groups of every size down to bf16's smallest values (no GPU)."""

import numpy as np
import pytest

from oracle import checkpoint as CK
from paper_2608_07524_amd import inputs as I


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_elements_move_by_at_most_the_stated_bounds(fmt):
    rng = np.random.default_rng(1)
    rows = 4000
    x = rng.standard_normal((rows, 32)) * np.exp2(rng.integers(-18, 1, (rows, 32)))
    x *= np.exp2(rng.integers(-133, 120, rows).astype(np.float64))[:, None]
    x = I.bf16_to_f64(I.bf16_bits(x.astype(np.float32)))
    vals, scales = CK.pack(x, fmt)
    k, top, moved = scales.astype(np.int64) - 127, np.max(np.abs(x), axis=1, keepdims=True), np.abs(vals - x)
    least = k == -126
    assert 100 < np.sum(least) < rows - 100
    if fmt == "int8":
        assert np.all(moved <= np.where(least, 2.0 ** -127, top / 127))
        assert np.any(moved > top / 127)  # (at the smallest scale only)
    else:
        # below the format's normal range half a step of it; at the smallest scale such
        # elements are multiples of 2^-133 and held exactly
        assert np.all(moved <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -17 * top))
        assert np.all((moved <= 2.0 ** -4 * np.abs(x)) | (np.abs(x) < 2.0 ** -13 * top))
