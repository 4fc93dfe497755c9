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


@pytest.mark.parametrize("n", [(1 << 30) + 1, (1 << 31) - 1])
def test_join_of_too_many_sequences_is_refused(n):
    """Beyond 2^30 the searches' and the launch's 32-bit counts would pass 2^31."""
    lib, at, size = P.load(), 1 << 20, C.c_size_t()
    d, w = N.GatedNormDescC(8, 64, n, at, 1.0, 1e-6, N.ACT_BF16, 0, 0), N.GatedNormPtrsC(None, 2 * at, None)
    assert lib.dcp_gated_norm_bwd_workspace_size(d, size) == N.DCP_ERR_UNSUPPORTED and "sequences" in P.last_error()
    assert lib.dcp_gated_norm_fwd(d, w, 3 * at, 4 * at, 5 * at, None, None, None, None, None,
                                  None) == N.DCP_ERR_UNSUPPORTED
    assert lib.dcp_gated_norm_bwd(d, w, 3 * at, None, N.KeptC(4 * at, None), None, None, None, None, 5 * at, None,
                                  N.GatedNormPtrsC(None, 6 * at, None), 7 * at, 1 << 40, None) == N.DCP_ERR_UNSUPPORTED
    ok = N.GatedNormDescC(8, 64, 1 << 30, at, 1.0, 1e-6, N.ACT_BF16, 0, 0)
    assert lib.dcp_gated_norm_bwd_workspace_size(ok, size) == N.DCP_OK
