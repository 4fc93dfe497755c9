"""The largest calls that a join's description admits."""

import ctypes as C

import pytest

import paper_2608_07524_amd as P
from paper_2608_07524_amd import _native as N


@pytest.mark.gpu
def test_join_of_almost_2_31_rows():
    """The last row counts: one launch holds fewer than 2^32 lanes.  The last rows equal a
    call on them alone."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rows, h, tail = (1 << 31) - 1, 8, 1000  # 34 GB a matrix
    x = torch.empty(rows, h, dtype=torch.bfloat16, device="cuda").normal_()
    g = torch.tensor([0.5, 1.0, 1.5, 2.0, -0.5, 0.25, 1.0, 0.75], dtype=torch.bfloat16, device="cuda")
    r = P.gated_norm_fwd(x, x, g, g)
    s = P.gated_norm_fwd(x[-tail:], x[-tail:], g, g)
    assert torch.equal(r.out[-tail:], s.out) and torch.equal(r.rstd_f[-tail:], s.rstd_f)
    b = P.gated_norm_bwd(x, f=x, rstd_f=r.rstd_f, post=g, gate=g, want_dx=False, df=r.out)
    c = P.gated_norm_bwd(x[-tail:], f=x[-tail:], rstd_f=s.rstd_f, post=g, gate=g, want_dx=False)
    assert torch.equal(b.df[-tail:], c.df)
    assert bool(torch.isfinite(b.dgate).all()) and bool(torch.isfinite(b.dpost).all())
