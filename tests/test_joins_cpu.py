"""8-bit checkpoints and gated joins on the CPU: the oracles against properties and
differences, and every refusal of the C ABI and of the binding before any
device call."""

import ctypes as C

import numpy as np
import pytest

import paper_2608_07524_amd as P
from oracle import checkpoint as CK
from oracle import join as J
from paper_2608_07524_amd import _native as N
from paper_2608_07524_amd import inputs as I

FAKE = 1 << 20  # an aligned address that is never dereferenced


# ---------------------------------------------------------------------------
# oracles

@pytest.mark.parametrize("fmt,step", [("int8", 2.0 ** -7), ("e4m3", 2.0 ** -4)])
def test_checkpoint_oracle_bounds(fmt, step):
    """Half a step of int8 is at most max / 127 < 2^-6.98 of the group's max, of
    e4m3 2^-4 of the value (2^-13 of the max at the least); packing again changes
    nothing; a group scales with powers of two."""
    rng = np.random.default_rng(1)
    x = I.bf16_to_f64(I.bf16_bits((rng.standard_normal((64, 72)) * np.exp(3 * rng.standard_normal((64, 1)))).astype(
        np.float32)))
    v, b = CK.pack(x, fmt)
    for g in range(3):
        part, got = x[:, 32 * g:32 * g + 32], v[:, 32 * g:32 * g + 32]
        top = np.abs(part).max(axis=1, keepdims=True)
        bound = top / 127 if fmt == "int8" else np.maximum(2.0 ** -4 * np.abs(part), 2.0 ** -17 * top)
        assert np.all(np.abs(got - part) <= bound)
    v2, b2 = CK.pack(v, fmt)
    assert np.array_equal(v, v2) and np.all(b2 <= b)
    v3, b3 = CK.pack(x * 2.0 ** 9, fmt)
    assert np.array_equal(v3, v * 2.0 ** 9) and np.array_equal(b3, b + 9)


def test_checkpoint_oracle_edges():
    x = np.zeros((3, 40))
    x[0, 0], x[0, 33] = np.inf, 127.0
    x[1, 5], x[1, 39] = 127.5, 2.0 ** -133
    v, b = CK.pack(x, "int8")
    assert np.all(np.isnan(v[0, :32])) and b[0, 0] == 255 and b[0, 1] == 127 and v[0, 33] == 127.0
    assert v[1, 5] == 128.0 and b[1, 0] == 128 and b[1, 1] == 1 and v[1, 39] == 0.0  # 127.5 does not fit 2^0
    v, b = CK.pack(np.array([[448.0, 17.0, 2.0 ** -10, 3 * 2.0 ** -10]]), "e4m3")
    assert b[0, 0] == 127 and v.tolist() == [[448.0, 16.0, 0.0, 2.0 ** -8]]  # ties to even
    assert len(CK.E4M3) == 127 and CK.E4M3[-1] == 448.0 and np.all(np.diff(CK.E4M3) > 0)


@pytest.mark.parametrize("post,gate,pre", [(1, "sequence", 1), (1, "shared", 1), (0, "sequence", 1), (1, None, 1),
                                           (0, None, 1), (1, "sequence", 0), (0, "shared", 0)])
def test_join_oracle_against_differences(post, gate, pre):
    rng = np.random.default_rng(7)
    h, cu = 6, np.array([0, 2, 2, 5])
    rows = int(cu[-1])
    r = lambda *s: rng.standard_normal(s)
    v = dict(x=r(rows, h), f=r(rows, h))
    if post:
        v["post"] = 1 + 0.3 * r(h)
    if gate:
        v["gate"] = r(3, h) if gate == "sequence" else r(h)
    if pre:
        v["pre"] = 1 + 0.3 * r(h)
    per = cu if gate == "sequence" else None
    dout, dy = r(rows, h), r(rows, h)

    def loss(**a):
        o = J.forward(cu=per, alpha=0.7, eps=1e-3, **a)
        return float(np.sum(dout * o["out"]) + (np.sum(dy * o["y"]) if pre else 0.0))

    o = J.forward(cu=per, alpha=0.7, eps=1e-3, **v)
    w = {n: v[n] for n in ("post", "gate", "pre") if n in v}
    g, _ = J.backward(dout, dy, v["f"], o["out"], o["rstd_f"], o["rstd_out"], cu=per, alpha=0.7, **w)
    if pre:
        assert np.allclose(g["y"], o["y"], rtol=1e-12)
    for n in v:
        num = np.zeros_like(v[n])
        for i in np.ndindex(v[n].shape):
            up, dn = v[n].copy(), v[n].copy()
            up[i] += 1e-5
            dn[i] -= 1e-5
            num[i] = (loss(**{**v, n: up}) - loss(**{**v, n: dn})) / 2e-5
        assert np.max(np.abs(num - g["d" + n])) < 1e-7, n
    if gate == "sequence":
        assert np.all(g["dgate"][1] == 0.0)  # the empty sequence


# ---------------------------------------------------------------------------
# refusals of the C ABI

@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), N.DCP_ERR_INVALID), (dict(rows=1 << 31), N.DCP_ERR_INVALID), (dict(cols=0), N.DCP_ERR_INVALID),
    (dict(cols=60, ld=64), N.DCP_ERR_UNSUPPORTED), (dict(ld=56), N.DCP_ERR_INVALID), (dict(ld=68), N.DCP_ERR_INVALID),
    (dict(fmt=3), N.DCP_ERR_INVALID), (dict(fmt=N.ACT_BF16), N.DCP_ERR_INVALID), (dict(x=None), N.DCP_ERR_INVALID),
    (dict(x=FAKE + 8), N.DCP_ERR_INVALID), (dict(codes=FAKE + 4), N.DCP_ERR_INVALID),
    (dict(scales=None), N.DCP_ERR_INVALID),
])
def test_act8_refusals(kw, code):
    lib = P.load()
    a = dict(rows=4, cols=64, fmt=N.ACT_INT8, ld=64, x=FAKE, codes=FAKE, scales=FAKE)
    a.update(kw)
    d = N.Act8DescC(a["rows"], a["cols"], a["fmt"], a["ld"])
    assert lib.dcp_act8_pack(C.byref(d), a["x"], a["codes"], a["scales"], None) == code
    assert lib.dcp_act8_unpack(C.byref(d), a["codes"], a["scales"], a["x"], None) == code and P.last_error()
    if a["fmt"] != N.ACT_BF16:
        assert lib.dcp_act8_gelu_bwd(C.byref(d), a["codes"], a["scales"], a["x"], FAKE, 2 * FAKE, None) == code


def test_act8_null_and_shared_buffers():
    lib = P.load()
    d = N.Act8DescC(4, 64, N.ACT_INT8, 64)
    assert lib.dcp_act8_pack(None, FAKE, FAKE, FAKE, None) == N.DCP_ERR_INVALID
    assert lib.dcp_act8_gelu_bwd(C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None) == N.DCP_ERR_INVALID  # du is a
    bf = N.Act8DescC(4, 64, N.ACT_BF16, 64)
    assert lib.dcp_act8_gelu_bwd(C.byref(bf), FAKE + 8, None, FAKE, FAKE, 2 * FAKE, None) == N.DCP_ERR_INVALID
    empty = N.Act8DescC(0, 64, N.ACT_INT8, 64)
    assert lib.dcp_act8_pack(C.byref(empty), None, None, None, None) == N.DCP_OK


def _join(rows=8, hidden=64, n_seqs=0, cu=None, alpha=1.0, eps=1e-6, fmt=N.ACT_BF16, f32=0, acc=0):
    return N.GatedNormDescC(rows, hidden, n_seqs, cu, alpha, eps, fmt, f32, acc)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), N.DCP_ERR_INVALID), (dict(rows=1 << 31), N.DCP_ERR_INVALID), (dict(hidden=0), N.DCP_ERR_INVALID),
    (dict(hidden=60), N.DCP_ERR_UNSUPPORTED), (dict(hidden=4104), N.DCP_ERR_UNSUPPORTED),
    (dict(n_seqs=2), N.DCP_ERR_INVALID), (dict(cu=FAKE), N.DCP_ERR_INVALID),
    (dict(n_seqs=-1, cu=FAKE), N.DCP_ERR_INVALID),
    (dict(n_seqs=2, cu=FAKE + 2), N.DCP_ERR_INVALID), (dict(alpha=float("inf")), N.DCP_ERR_INVALID),
    (dict(eps=-1.0), N.DCP_ERR_INVALID), (dict(eps=float("nan")), N.DCP_ERR_INVALID), (dict(fmt=3), N.DCP_ERR_INVALID),
    (dict(f32=2), N.DCP_ERR_INVALID), (dict(acc=-1), N.DCP_ERR_INVALID),
])
def test_join_descriptor_refusals(kw, code):
    lib = P.load()
    d, w = _join(**kw), N.GatedNormPtrsC(FAKE, FAKE, FAKE)
    n = C.c_size_t()
    assert lib.dcp_gated_norm_bwd_workspace_size(C.byref(d), C.byref(n)) == code and P.last_error()
    assert lib.dcp_gated_norm_fwd(C.byref(d), C.byref(w), FAKE, FAKE, FAKE, 2 * FAKE, FAKE, FAKE, None, None,
                                  None) == code
    assert lib.dcp_gated_norm_bwd(C.byref(d), C.byref(w), *([FAKE] * 2), None, None, FAKE, FAKE, FAKE, 2 * FAKE, None,
                                  C.byref(w), FAKE, 1 << 30, None) == code


def test_join_forward_refusals():
    lib = P.load()
    d, w = _join(), N.GatedNormPtrsC(FAKE, FAKE, FAKE)

    def call(desc=d, wt=w, x=FAKE, f=FAKE, out=FAKE, y=2 * FAKE, rf=FAKE, ro=FAKE, kf=None, ko=None):
        return lib.dcp_gated_norm_fwd(C.byref(desc), None if wt is None else C.byref(wt), x, f, out, y, rf, ro, kf, ko,
                                      None)

    bad = N.DCP_ERR_INVALID
    assert call(wt=None) == bad and call(x=None) == bad and call(f=FAKE + 8) == bad and call(y=None) == bad
    assert call(y=FAKE) == bad  # out's buffer
    assert call(rf=None) == bad and call(ro=None) == bad
    assert call(wt=N.GatedNormPtrsC(FAKE + 2, FAKE, FAKE)) == bad
    assert call(wt=N.GatedNormPtrsC(FAKE, FAKE, None)) == bad  # y without pre
    assert call(desc=_join(n_seqs=2, cu=FAKE), wt=N.GatedNormPtrsC(FAKE, None, FAKE)) == bad  # offsets, no gate
    kept = N.KeptC(FAKE, FAKE)
    assert call(kf=C.byref(kept)) == bad  # in bf16 f itself is kept
    i8 = _join(fmt=N.ACT_INT8)
    assert call(desc=i8, kf=C.byref(N.KeptC(FAKE, None))) == bad
    assert call(desc=i8, ko=C.byref(N.KeptC(FAKE + 4, FAKE))) == bad


def test_join_backward_refusals():
    lib = P.load()
    n = C.c_size_t()
    d = _join(fmt=N.ACT_E4M3)
    assert lib.dcp_gated_norm_bwd_workspace_size(C.byref(d), C.byref(n)) == 0 and n.value >= 2 * 4 * 64
    assert lib.dcp_gated_norm_bwd_workspace_size(C.byref(d), None) == N.DCP_ERR_INVALID
    w, k = N.GatedNormPtrsC(FAKE, FAKE, FAKE), N.KeptC(FAKE, FAKE)
    grads = N.GatedNormPtrsC(FAKE, FAKE + 256, FAKE + 512)

    def call(wt=w, dout=FAKE, dy=FAKE, f=k, out=k, rf=FAKE, ro=FAKE, dx=FAKE, df=2 * FAKE, y=None, g=grads, ws=FAKE,
             size=n.value):
        ref = lambda s: None if s is None else C.byref(s)
        return lib.dcp_gated_norm_bwd(C.byref(d), ref(wt), dout, dy, ref(f), ref(out), rf, ro, dx, df, y, ref(g), ws,
                                      size, None)

    bad = N.DCP_ERR_INVALID
    for kw in (dict(wt=None), dict(g=None), dict(dy=None), dict(dy=FAKE + 4), dict(dout=FAKE + 8), dict(f=None),
               dict(out=None), dict(f=N.KeptC(FAKE, None)), dict(out=N.KeptC(FAKE + 1, FAKE)), dict(rf=None),
               dict(ro=None), dict(df=None), dict(dx=2 * FAKE), dict(y=FAKE), dict(y=FAKE + 8),
               dict(g=N.GatedNormPtrsC(FAKE, None, 2 * FAKE)), dict(g=N.GatedNormPtrsC(FAKE, 2 * FAKE, FAKE + 1)),
               dict(g=N.GatedNormPtrsC(FAKE, FAKE, 2 * FAKE)), dict(g=N.GatedNormPtrsC(FAKE, 2 * FAKE, 2 * FAKE)),
               dict(wt=N.GatedNormPtrsC(FAKE, FAKE, None), g=N.GatedNormPtrsC(FAKE, 2 * FAKE, None)),  # dy without pre
               dict(wt=N.GatedNormPtrsC(FAKE, FAKE, None), g=N.GatedNormPtrsC(FAKE, 2 * FAKE, None), dy=None,
                    dout=None)):
        assert call(**kw) == bad, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(size=n.value - 1)):
        assert call(**kw) == N.DCP_ERR_WORKSPACE, kw


# ---------------------------------------------------------------------------
# refusals of the binding

def test_binding_refuses_before_any_call():
    import torch
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    x, g = bf(6, 64), bf(64)
    with pytest.raises(ValueError, match="device"):
        P.act8_pack(x)
    with pytest.raises(ValueError, match="device"):
        P.gated_norm_fwd(x, x, post=g)
    codes, scales = torch.zeros(6, 64, dtype=torch.int8), torch.zeros(6, 2, dtype=torch.uint8)
    cases = [lambda: P.act8_pack(x.float()), lambda: P.act8_pack(x.t()), lambda: P.act8_pack(bf(64)),
             lambda: P.act8_pack(x, "int4"), lambda: P.act8_unpack(codes, scales[:, :1]),
             lambda: P.act8_unpack(x, scales), lambda: P.act8_unpack(codes.t(), scales),
             lambda: P.act8_unpack(codes, scales.int()), lambda: P.act8_gelu_bwd(codes, scales, x[:5]),
             lambda: P.act8_gelu_bwd(codes, None, x), lambda: P.act8_gelu_bwd(x, scales, x),
             lambda: P.act8_gelu_bwd(codes, scales, bf(6, 128)[:, ::2]),
             lambda: P.gated_norm_fwd(x, x[:5]), lambda: P.gated_norm_fwd(x, x.float()),
             lambda: P.gated_norm_fwd(x, x, y=x), lambda: P.gated_norm_fwd(x, x, keep_f="int8", keep_out="e4m3"),
             lambda: P.gated_norm_fwd(x, x, keep_f="bf16"), lambda: P.gated_norm_fwd(bf(64), bf(64)),
             lambda: P.gated_norm_bwd(x, x), lambda: P.gated_norm_bwd(None), lambda: P.gated_norm_bwd(x, pre=g),
             lambda: P.gated_norm_bwd(x, post=g), lambda: P.gated_norm_bwd(x, f=x[:5], post=g),
             lambda: P.gated_norm_bwd(x, x, (codes, scales), x, post=g, pre=g),
             lambda: P.gated_norm_bwd(x, x, x, x, torch.zeros(5), torch.zeros(6), post=g, pre=g),
             lambda: P.gated_norm_bwd(x, want_y=True)]
    for i, c in enumerate(cases):
        with pytest.raises(ValueError) as e:
            c()
        assert "must be on a CUDA" not in str(e.value), (i, str(e.value))


def test_binding_refuses_weights_and_offsets():
    import torch
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    dev = torch.device("cpu")
    ok = dict(post=None, gate=None, pre=None, cu_seqlens=None)
    cases = [dict(post=bf(63)), dict(post=bf(64).float()), dict(pre=bf(128)[::2]), dict(gate=bf(2, 64)),
             dict(cu_seqlens=[0, 6]), dict(gate=bf(2, 64), cu_seqlens=[0, 6]), dict(gate=bf(1, 64), cu_seqlens=[0, 7]),
             dict(gate=bf(2, 64), cu_seqlens=[0, 4, 3]), dict(gate=bf(1, 64), cu_seqlens=[1, 6]),
             dict(gate=bf(1, 64), cu_seqlens=[0])]
    for kw in cases:
        with pytest.raises(ValueError):
            N._join_weights(torch, (6, 64), *{**ok, **kw}.values(), dev)
    n, cu = N._join_weights(torch, (6, 64), None, bf(3, 64), None, [0, 2, 2, 5], dev)
    assert n == 3 and cu.dtype == torch.int32 and cu.tolist() == [0, 2, 2, 5]
    assert N._join_weights(torch, (6, 64), None, bf(64), None, None, dev) == (0, None)
