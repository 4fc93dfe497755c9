"""The transformer block on the CPU: its oracle against finite differences and
against the layer's, its sizes, and its refusals before any device call."""

import ctypes as C

import numpy as np
import pytest

import paper_2608_07524_amd as P
from oracle import block as B
from oracle import layer as LY
from paper_2608_07524_amd import _native as N

FAKE = 1 << 20


def _weights(rng, h, post, gates):
    W = {}
    for n, s in P.block_param_shapes(h, post, gates).items():
        v = rng.standard_normal(s)
        W[n] = 1 + 0.2 * v if n.startswith(("norm", "post")) else v if "gate" in n else v / np.sqrt(s[0])
    return W


@pytest.mark.parametrize("post,gates,causal", [(True, 3, True), (True, 1, False), (False, 3, False), (True, 0, True),
                                               (False, 0, False)])
def test_block_oracle_against_differences(post, gates, causal):
    rng = np.random.default_rng(3)
    H, D, cu = 2, 4, [0, 3, 3, 7]
    h, T = H * D, cu[-1]
    W = _weights(rng, h, post, gates)
    x, dout = rng.standard_normal((T, h)), rng.standard_normal((T, h))
    args = (cu, H, D, 0.5, causal, 1e-3, 0.75)
    out, kept = B.forward(x, W, *args)
    dx, g = B.backward(dout, x, W, kept, *args)
    assert set(g) == set(W)
    loss = lambda x_, W_: float(np.sum(dout * B.forward(x_, W_, *args)[0]))

    def check(name, value, grad, at):
        for i in rng.permutation(value.size)[:12]:
            up, dn = value.copy().reshape(-1), value.copy().reshape(-1)
            up[i] += 1e-5
            dn[i] -= 1e-5
            num = (at(up.reshape(value.shape)) - at(dn.reshape(value.shape))) / 2e-5
            assert abs(num - grad.reshape(-1)[i]) < 1e-6, (name, i)

    check("x", x, dx, lambda a: loss(a, W))
    for n in W:
        check(n, W[n], g[n], lambda a: loss(x, {**W, n: a}))


def test_plain_block_is_the_layer():
    rng = np.random.default_rng(4)
    H, D, cu = 2, 8, [0, 5, 11]
    W = _weights(rng, H * D, False, 0)
    x, dout = rng.standard_normal((11, 16)), rng.standard_normal((11, 16))
    out, kept = B.forward(x, W, cu, H, D, 0.3, True, 1e-6, 1.0)
    dx, g = B.backward(dout, x, W, kept, cu, H, D, 0.3, True, 1e-6, 1.0)
    ref, cache = LY.layer_forward(x, W, cu, H, D, 0.3, True, 1e-6)
    rdx, rg = LY.layer_backward(dout, W, cache, cu, H, D, 0.3, True)
    assert np.allclose(out, ref, rtol=1e-12, atol=1e-12) and np.allclose(dx, rdx, rtol=1e-9, atol=1e-11)
    for n in W:
        assert np.allclose(g[n], rg[n], rtol=1e-9, atol=1e-10), n


def _desc(cu=(0, 30, 64), H=2, D=64, eps=1e-6, fmt=N.ACT_INT8, post=1, gate=N.GATE_SHARED, dev_cu=None, alpha=1.0,
          T=None):
    a = np.asarray(cu, dtype=np.int32)
    d = N.AttnDesc(a.size - 1, a.ctypes.data_as(C.POINTER(C.c_int32)), int(a[-1]) if T is None else T, H, D, 0.125, 0)
    L = N.LayerDescC(C.pointer(d), eps)
    return N.BlockDescC(C.pointer(L), fmt, post, gate, dev_cu, alpha), (a, d, L)


def test_block_sizes():
    """Per token and hidden column: 11 (9 without norms and gates) elements kept, at
    1 + 1/32 bytes, or 2, and o always at 2; the layer's stash has 30 bytes."""
    lib = P.load()
    s, f, b = C.c_size_t(), C.c_size_t(), C.c_size_t()
    sizes = {}
    for fmt in (N.ACT_BF16, N.ACT_INT8, N.ACT_E4M3):
        for post, gate in ((0, N.GATE_NONE), (1, N.GATE_SHARED), (0, N.GATE_SHARED)):
            d, keep = _desc(cu=(0, 4096), H=16, D=72, fmt=fmt, post=post, gate=gate)
            assert lib.dcp_block_sizes(C.byref(d), C.byref(s), C.byref(f), C.byref(b)) == 0
            sizes[fmt, post, gate] = s.value
            n = ((10 if post or gate else 8) * (2.0 if fmt == N.ACT_BF16 else 33 / 32) + 2.0) * 4096 * 1152
            rows = 4 * 4096 * (16 + 3)
            assert n + rows <= s.value <= n + rows + 24 * 256
            assert f.value > s.value and b.value > f.value
    layer = C.c_size_t()
    assert lib.dcp_layer_sizes(d.layer, C.byref(layer), None, None) == 0
    assert layer.value > 2.9 * sizes[N.ACT_INT8, 0, N.GATE_NONE]


@pytest.mark.parametrize("kw,code", [
    (dict(fmt=3), N.DCP_ERR_INVALID), (dict(fmt=-1), N.DCP_ERR_INVALID), (dict(post=2), N.DCP_ERR_INVALID),
    (dict(gate=3), N.DCP_ERR_INVALID), (dict(gate=N.GATE_SEQUENCE), N.DCP_ERR_INVALID),
    (dict(dev_cu=FAKE), N.DCP_ERR_INVALID),
    (dict(gate=N.GATE_SEQUENCE, dev_cu=FAKE + 2), N.DCP_ERR_INVALID), (dict(alpha=float("nan")), N.DCP_ERR_INVALID),
    (dict(T=70), N.DCP_ERR_INVALID), (dict(eps=-1.0), N.DCP_ERR_INVALID), (dict(H=64, D=128), N.DCP_ERR_UNSUPPORTED),
    (dict(D=96), N.DCP_ERR_UNSUPPORTED),
])
def test_block_descriptor_refusals(kw, code):
    lib = P.load()
    d, keep = _desc(**kw)
    s = C.c_size_t()
    assert lib.dcp_block_sizes(C.byref(d), C.byref(s), None, None) == code and P.last_error()
    w = N.BlockWeightsC(N.LayerWeightsC(*([FAKE] * 8)), FAKE, FAKE, FAKE, FAKE)
    assert lib.dcp_block_fwd(C.byref(d), C.byref(w), FAKE, FAKE, None, FAKE, 1 << 40, None) == code
    assert lib.dcp_block_bwd(C.byref(d), C.byref(w), FAKE, FAKE, FAKE, C.byref(w), None, FAKE, 1 << 40, None) == code
    assert lib.dcp_block_sizes(None, C.byref(s), None, None) == N.DCP_ERR_INVALID


def test_block_call_refusals():
    lib = P.load()
    d, keep = _desc()
    f, b = C.c_size_t(), C.c_size_t()
    assert lib.dcp_block_sizes(C.byref(d), None, C.byref(f), C.byref(b)) == 0
    layer = N.LayerWeightsC(*([FAKE] * 8))

    def grads(norm2=FAKE + 16, joins=(FAKE, FAKE + 32, FAKE, FAKE + 32)):
        return N.BlockWeightsC(N.LayerWeightsC(FAKE, FAKE, FAKE, FAKE, FAKE, norm2, FAKE, FAKE), *joins)

    w = N.BlockWeightsC(layer, FAKE, FAKE, FAKE, FAKE)

    def fwd(w=w, x=FAKE, out=FAKE, stash=None, ws=FAKE, size=f.value):
        return lib.dcp_block_fwd(C.byref(d), None if w is None else C.byref(w), x, out, stash, ws, size, None)

    def bwd(w=w, x=FAKE, dout=FAKE, dx=FAKE, g=grads(), stash=None, ws=FAKE, size=b.value):
        ref = lambda v: None if v is None else C.byref(v)
        return lib.dcp_block_bwd(C.byref(d), ref(w), x, dout, dx, ref(g), stash, ws, size, None)

    bad = N.DCP_ERR_INVALID
    for joins in ((None, FAKE, FAKE, FAKE), (FAKE, FAKE, FAKE, None), (FAKE + 8, FAKE, FAKE, FAKE)):
        assert fwd(w=N.BlockWeightsC(layer, *joins)) == bad and bwd(w=N.BlockWeightsC(layer, *joins)) == bad
    assert fwd(w=None) == bad and fwd(x=None) == bad and fwd(out=FAKE + 8) == bad and fwd(stash=FAKE + 16) == bad
    assert fwd(ws=None) == fwd(size=f.value - 1) == fwd(ws=FAKE + 64) == N.DCP_ERR_WORKSPACE
    assert bwd(dout=None) == bad and bwd(g=None) == bad and bwd(stash=FAKE + 16) == bad
    assert bwd(g=grads(joins=(FAKE, None, FAKE, FAKE))) == bad
    assert bwd(g=grads(norm2=FAKE)) == bad  # post1's buffer
    assert bwd(g=grads(joins=(FAKE, FAKE + 16, FAKE, FAKE + 32))) == bad  # gate1's is norm2's
    assert bwd(g=grads(joins=(FAKE, FAKE + 32, FAKE, FAKE))) == bad
    assert bwd(size=b.value - 1) == N.DCP_ERR_WORKSPACE
    import torch
    if not torch.cuda.is_available():
        assert fwd() == N.DCP_ERR_HIP and bwd() == N.DCP_ERR_HIP


def test_block_binding_refusals():
    import torch
    h, cu = 128, [0, 5, 9]

    def make(post=True, gates=2, **change):
        W = {n: torch.zeros(s, dtype=torch.bfloat16) for n, s in P.block_param_shapes(h, post, gates).items()}
        W.update(change)
        G = {n: torch.zeros(t.shape, dtype=torch.float32) for n, t in W.items()}
        return W, G

    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    W, G = make()
    with pytest.raises(ValueError, match="device"):
        P.Block(W, G, cu, 2, 64)
    cases = [make(gates=3), make(gate2=bf(1, h)), make(wq=bf(h, h + 8)), make(norm1=bf(h).float()), make(), (W, {**G, "wq": G["wq"].bfloat16()}), (W, {n: g for n, g in G.items() if n != "post1"}),
             ({n: w for n, w in W.items() if n != "post2"}, G)]
    cases[4][0]["wo"] = bf(h, 2 * h)[:, ::2]
    for i, (w, g) in enumerate(cases):
        with pytest.raises(ValueError) as e:
            P.Block(w, g, cu, 2, 64)
        assert "must be on a CUDA" not in str(e.value), i
    with pytest.raises(ValueError):
        P.Block(W, G, cu, 2, 64, stash_format="int4")


def test_smaller_stash_recomputes_fewer_layers():
    """The planner given a layer's and a block's m (same times, one budget): in 8 bits
    fewer layers are recomputed."""
    lib = P.load()
    layer, b8 = C.c_size_t(), C.c_size_t()
    d, keep = _desc(cu=(0, 16384), H=16, D=72, post=0, gate=N.GATE_NONE)
    assert lib.dcp_layer_sizes(d.layer, C.byref(layer), None, None) == 0
    assert lib.dcp_block_sizes(C.byref(d), C.byref(b8), None, None) == 0
    m_inp = 2 * 16384 * 1152

    def recomputed(m):
        # (one device, one micro-batch: the budget holds 10 of 28 layers' bf16 stashes)
        p = P.plan([16384], [(16384, 10 ** 6, 2 * 10 ** 6, m, m_inp)], 28, 0, 0, 10 * layer.value + 28 * m_inp,
                   sp_cands=(1,), b_max=1)
        return p.recompute_layers[0]

    assert recomputed(layer.value) == 18 and recomputed(b8.value) == 0
