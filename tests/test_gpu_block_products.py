"""Blocks with a bf16 stash against the float64 oracle on both sides of the sizes from which
W_down^T and GELU's backward are the library's product and a pass, instead of one kernel."""

import pytest

from gpu_util import GRAD_TOL
from test_gpu_block import _errors, _setup, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,D,lengths", [(8, 128, [600, 420]), (8, 128, [600, 430]), (8, 128, [1100]), (16, 72, [1100]),
                                         (10, 128, [520])])
def test_block_on_both_sides_of_the_rule(torch, H, D, lengths):  # noqa: F811
    block, cu, W, host, dev = _setup(torch, lengths, H, D, True, True, len(lengths), "bf16")
    errs = _errors(torch, block, cu, W, host, dev, H, D, True, "bf16", 1.0)
    assert max(errs.values()) <= GRAD_TOL, errs
