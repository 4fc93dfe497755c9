"""Calls whose outputs share memory with another buffer, refused by the C ABI before any
device call (no GPU)."""

import ctypes as C

import pytest

import paper_2608_07524_amd as P
from paper_2608_07524_amd import _native as N

ROWS, H = 64, 64
MATRIX, CODES, SCALES, ROW = 2 * ROWS * H, ROWS * H, ROWS * 2, 4 * ROWS
SPOT = 1 << 20  # addresses that nothing reads: every buffer in a place of its own, this far apart


def _places(*names):
    return {n: SPOT * (i + 1) for i, n in enumerate(names)}


def _forward(**moved):
    at = _places("x", "f", "out", "y", "rstd_f", "rstd_out", "fc", "fs", "oc", "os", "post", "gate", "pre", "cu")
    at.update(moved)
    d = N.GatedNormDescC(ROWS, H, 3, at["cu"], 1.0, 1e-6, N.ACT_INT8, 0, 0)
    w = N.GatedNormPtrsC(at["post"], at["gate"], at["pre"])
    return P.load().dcp_gated_norm_fwd(d, w, at["x"], at["f"], at["out"], at["y"], at["rstd_f"], at["rstd_out"],
                                       N.KeptC(at["fc"], at["fs"]), N.KeptC(at["oc"], at["os"]), None)


def _backward(f32=1, fmt=N.ACT_INT8, **moved):
    at = _places("dout", "dy", "fc", "fs", "oc", "os", "rstd_f", "rstd_out", "dx", "df", "y", "dpost", "dgate", "dpre",
                 "ws", "post", "gate", "pre", "cu")
    at.update(moved)
    d = N.GatedNormDescC(ROWS, H, 3, at["cu"], 1.0, 0.0, fmt, f32, 0)
    n = C.c_size_t()
    assert P.load().dcp_gated_norm_bwd_workspace_size(d, n) == 0 and n.value < SPOT
    return P.load().dcp_gated_norm_bwd(d, N.GatedNormPtrsC(at["post"], at["gate"], at["pre"]), at["dout"], at["dy"],
                                       N.KeptC(at["fc"], at["fs"]), N.KeptC(at["oc"], at["os"]), at["rstd_f"],
                                       at["rstd_out"], at["dx"], at["df"], at["y"],
                                       N.GatedNormPtrsC(at["dpost"], at["dgate"], at["dpre"]), at["ws"], n.value, None)


F = _places("x", "f", "out", "y", "rstd_f", "rstd_out", "fc", "fs", "oc", "os", "post", "gate", "pre", "cu")


@pytest.mark.parametrize("moved", [
    dict(oc=F["fc"]), dict(os=F["fs"]), dict(rstd_out=F["rstd_f"]), dict(fc=F["x"]), dict(oc=F["f"] + CODES),
    dict(fs=F["out"]), dict(fs=F["fc"] + CODES - 1), dict(out=F["x"] + 2 * H), dict(out=F["f"] - 2 * H),
    dict(y=F["out"] + 2 * H), dict(y=F["x"] + 16, out=F["f"]), dict(rstd_f=F["y"]), dict(rstd_out=F["cu"]),
    dict(out=F["gate"] - MATRIX + 16), dict(y=F["pre"]), dict(fc=F["post"] + 2 * H - 8),
])
def test_join_forward_refuses_shared_memory(moved):
    assert _forward(**moved) == N.DCP_ERR_INVALID and "shares memory" in P.last_error()


B = _places("dout", "dy", "fc", "fs", "oc", "os", "rstd_f", "rstd_out", "dx", "df", "y", "dpost", "dgate", "dpre",
            "ws", "post", "gate", "pre", "cu")


@pytest.mark.parametrize("moved", [
    dict(dx=B["dy"]), dict(df=B["dy"]), dict(y=B["dy"]),  # fp32 rows that other teams have not read
    dict(dx=B["dy"] + MATRIX), dict(f32=0, dx=B["dy"] + 2 * H), dict(dx=B["dout"] + 2 * H), dict(df=B["dout"] - 16),
    dict(dx=B["fc"]), dict(y=B["oc"]), dict(df=B["fs"] - MATRIX + 16), dict(dx=B["df"] + 2 * H),
    dict(fmt=N.ACT_BF16, df=B["fc"] + 16), dict(fmt=N.ACT_BF16, dx=B["oc"] + MATRIX - 16),
    dict(dpost=B["dgate"] + 4 * H), dict(dpre=B["dpost"] + 4 * H - 4), dict(dpre=B["rstd_out"]), dict(ws=B["dout"]),
    dict(ws=B["dx"] + MATRIX // 2), dict(dgate=B["ws"] + 256), dict(dpost=B["post"]), dict(dgate=B["cu"]),
])
def test_join_backward_refuses_shared_memory(moved):
    assert _backward(**moved) == N.DCP_ERR_INVALID and "shares memory" in P.last_error()


def test_checkpoints_refuse_shared_memory():
    lib = P.load()
    x, codes, scales, du, a = (SPOT * i for i in range(1, 6))
    for ld in (H, 3 * H):
        d = N.Act8DescC(ROWS, H, N.ACT_E4M3, ld)
        wide = 2 * ld * (ROWS - 1) + 2 * H  # bytes from x's first element to its last
        for c, s in ((x, scales), (x + wide - 8, scales), (x - CODES + 8, scales), (codes, x), (codes, codes + CODES - 1)):
            assert lib.dcp_act8_pack(d, x, c, s, None) == N.DCP_ERR_INVALID and "shares memory" in P.last_error()
        for c, s in ((x, scales), (x + wide - 8, scales), (x - CODES + 8, scales), (codes, x)):
            assert lib.dcp_act8_unpack(d, c, s, x, None) == N.DCP_ERR_INVALID and "shares memory" in P.last_error()
        for to in ((codes, a), (du, codes), (du, du + 16), (x + 16, a), (du, x - 2 * ld + 16), (x, x + 2 * H - 16)):
            assert lib.dcp_act8_gelu_bwd(d, codes, scales, x, *to, None) == N.DCP_ERR_INVALID
            assert "shares memory" in P.last_error(), to
    b = N.Act8DescC(ROWS, H, N.ACT_BF16, H)
    assert lib.dcp_act8_gelu_bwd(b, codes, None, x, codes + 16, a, None) == N.DCP_ERR_INVALID
    assert "shares memory" in P.last_error()
