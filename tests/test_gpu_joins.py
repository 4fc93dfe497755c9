"""GPU parity of the 8-bit activation checkpoints and of the gated, normed join
against the float64 oracles.

Tolerances.  Codes, scale bytes and read-back values: equal.  A bf16 result is
rounded once (half a step, 2^-8 of the value) from an fp32 computation whose
error is relative to the magnitudes it adds: a row's sum passes at most 8 values
a lane, 2-3 chunks, 6 lane steps and 4 wavefronts, a result takes some ten further
operations, in all fewer than 64 roundings of 2^-24: 2^-18 of the terms' sum, plus
the hardware's exp, reciprocal and reciprocal root (1 ulp each, 2^-23, and e^x's
argument below 2^8 with 2^-24 of itself: 2^-16).  2^-15 of the magnitudes covers
both.  Weight gradients are fp32 sums over rows: up to 128 rows in a lane, 32 teams,
and partial rows 32 apart in eight running sums, below 2^9 roundings for the sizes
here: 2^-15 of the sum of magnitudes; where the terms come from bf16 inputs
nothing else is lost."""

import numpy as np
import pytest

from oracle import checkpoint as CK
from oracle import join as J
from oracle import layer as LY
from paper_2608_07524_amd import inputs as I

from gpu_util import to_bits, to_device

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
SUM = 2.0 ** -15


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_07524_amd as P
    P.load()
    return t


@pytest.fixture(scope="module")
def P(torch):
    import paper_2608_07524_amd as P
    return P


def _bits(a):
    return I.bf16_bits(np.asarray(a, dtype=np.float32))


def _f64(t):
    return I.bf16_to_f64(to_bits(t))


def _hold(torch, x64, fmt):
    """A checkpoint on the device, made by the oracle."""
    vals, scales = CK.pack(x64, fmt)
    s = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)[:, :x64.shape[1]]
    dtype = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    return vals, (torch.from_numpy(vals / s).to(torch.float32).to(dtype).cuda(), torch.from_numpy(scales).cuda())


def _close(name, got, ref, mag, rel):
    over = np.abs(got - ref) - rel * np.abs(ref) - SUM * mag
    i = np.unravel_index(np.argmax(over), over.shape) if over.size else None
    assert over.size == 0 or over[i] <= 0, (name, i, got[i], ref[i], mag[i] if np.ndim(mag) else mag)


# ---------------------------------------------------------------------------
# checkpoints

def _awkward(rng, rows, cols):
    """Values of every size, zeros, groups at the borders of a scale, infinities and NaN."""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, 1)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    x[rng.random((rows, cols)) < 0.02] *= 64
    x[0] = 0.0
    if rows > 8:
        x[1] = 127.0 * rng.integers(-1, 2, cols)
        x[2] = 127.5 * rng.integers(-1, 2, cols)
        x[3] = 448.0 * rng.integers(-1, 2, cols) / (1 + rng.integers(0, 9, cols))
        x[4] = 450.0 * rng.integers(-1, 2, cols) / (1 + rng.integers(0, 9, cols))
        x[5] = np.exp2(rng.integers(-133, -110, cols).astype(np.float64))
        x[6] = 3.3e38 * rng.random(cols)
        x[7, 0], x[7, cols - 1] = np.inf, np.nan
        x[8] = rng.integers(-254, 255, cols) / 2.0  # halves: ties
        x[8, ::32] = 127.0
    return x


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("rows,cols,ld", [(1, 8, 8), (3, 32, 32), (37, 72, 72), (429, 256, 256), (16, 40, 120),
                                          (65, 1152, 3456), (300, 1152, 1152), (2, 4608, 4608), (1000, 24, 32)])
def test_pack_and_unpack(torch, P, fmt, rows, cols, ld):
    rng = np.random.default_rng(rows * cols)
    wide = np.full((rows, ld), 7.0)
    wide[:, :cols] = _awkward(rng, rows, cols)
    bits = _bits(wide)
    x = to_device(torch, bits)[:, :cols]
    vals, scales = CK.pack(I.bf16_to_f64(bits)[:, :cols], fmt)
    codes, s = P.act8_pack(x, fmt)
    back = P.act8_unpack(codes, s)
    assert np.array_equal(s.cpu().numpy(), scales)
    # exact in bf16, but for a value that was rounded up to 2^128 (from 1.9375 2^127 in
    # e4m3, from 1.984375 2^127 in int8), which bf16 holds as infinity
    with np.errstate(over="ignore"):
        want = I.bf16_to_f64(_bits(vals))
    assert np.array_equal(np.where(np.isinf(want), np.copysign(2.0 ** 128, want), want), vals, equal_nan=True)
    assert np.array_equal(_f64(back), want, equal_nan=True)
    # (NaN groups hold codes 0)
    held = np.where(np.isnan(vals), 0.0, vals / np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, axis=1)[:, :cols])
    assert np.array_equal(codes.float().cpu().numpy(), held)
    if ld > cols:  # into a slice: the columns beside it stay
        out = torch.full((rows, ld), 7.0, dtype=torch.bfloat16, device="cuda")
        P.act8_unpack(codes, s, out=out[:, :cols])
        assert np.array_equal(_f64(out)[:, :cols], want, equal_nan=True) and bool((out[:, cols:] == 7.0).all())


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("rows,cols", [(1, 8), (5, 72), (429, 1024), (33, 4608)])
def test_gelu_backward(torch, P, fmt, rows, cols):
    rng = np.random.default_rng(rows + cols)
    u = 3.0 * rng.standard_normal((rows, cols))
    u[0, :4] = [0.0, 40.0, -40.0, -5.0]
    da = rng.standard_normal((rows, cols))
    ub, db = _bits(u), _bits(da)
    u64, d64 = I.bf16_to_f64(ub), I.bf16_to_f64(db)
    if fmt == "bf16":
        args = (to_device(torch, ub), None)
    else:
        u64, args = _hold(torch, u64, fmt)
    # (1 + tanh w) / 2 = 1 / (1 + e^(-2w)): the oracle's 1 + tanh w cancels, with an
    # error of 2^-53, where u is far below 0 and a small
    w = np.sqrt(2.0 / np.pi) * (u64 + 0.044715 * u64 ** 3)
    with np.errstate(over="ignore"):
        act, slope = u64 / (1.0 + np.exp(-2.0 * w)), LY.gelu_grad(u64)
    assert np.max(np.abs(act - LY.gelu(u64))) <= 40 * 2.0 ** -52
    da_t = to_device(torch, db)
    du, a = P.act8_gelu_bwd(*args, da_t)
    # s and 1 - s are formed from fp32 exponentials: their errors are relative to 1 in
    # the slope (times |u| <= 16 where it is not 0 or 1), to the value in a; below
    # 2^-126 (u under -9.8) fp32 may flush to zero
    _close("a", _f64(a), act, np.abs(act) + 2.0 ** -100, BF16)
    _close("du", _f64(du), d64 * slope, np.abs(d64) * (1.0 + np.minimum(np.abs(u64), 16.0)) * 2.0 ** -4, BF16)
    again, _ = P.act8_gelu_bwd(*args, da_t, du=da_t)  # in da's place
    assert np.array_equal(to_bits(again), to_bits(du))


def test_gelu_backward_of_extreme_inputs(torch, P):
    u = torch.tensor([[1e20, -1e20, 3e38, -3e38, 12.0, -12.0, float("nan"), 0.0]], dtype=torch.bfloat16, device="cuda")
    du, a = P.act8_gelu_bwd(u, None, torch.ones_like(u))
    assert du[0, :6].tolist() == [1.0, 0.0, 1.0, 0.0, 1.0, 0.0] and du[0, 7] == 0.5 and bool(du[0, 6].isnan())
    assert a[0, 0] == u[0, 0] and a[0, 1] == 0 and a[0, 2] == u[0, 2] and a[0, 3] == 0 and bool(a[0, 6].isnan())


def test_checkpoints_of_more_than_2_31_elements(torch, P):
    """Element offsets, and the count of 8-column pieces, beyond 32 bits' reach."""
    rows, cols = 270_000, 8192  # 2.2e9 elements
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_()
    codes, s = P.act8_pack(x)
    back = P.act8_unpack(codes, s)
    for lo in (0, rows // 2, rows - 300):
        c, b = P.act8_pack(x[lo:lo + 300])
        assert torch.equal(c, codes[lo:lo + 300]) and torch.equal(b, s[lo:lo + 300])
        assert torch.equal(P.act8_unpack(c, b), back[lo:lo + 300])


def test_checkpoints_of_more_than_2_31_pieces(torch, P):
    """More 8-column pieces than one launch counts: the rest is a second one."""
    rows, cols = 131_080, 131_072  # 2^31 + 131,072 pieces; 34 GB, read back in place
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[:9].normal_()
    x[9:-18] = 1.0
    x[-18:] = x[:9].repeat(2, 1)
    want = x[:9].clone()
    codes, s = P.act8_pack(x)
    P.act8_unpack(codes, s, out=x)
    c, b = P.act8_pack(want)
    held = P.act8_unpack(c, b)
    for lo in (0, rows - 18, rows - 9):
        assert torch.equal(codes[lo:lo + 9], c) and torch.equal(s[lo:lo + 9], b) and torch.equal(x[lo:lo + 9], held)
    assert bool((x[65_000:65_010] == 1.0).all())


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
def test_gelu_backward_in_wider_matrices(torch, P, fmt):
    """The C call on slices: row strides of da, du, a (and a bf16 u) beyond cols."""
    from paper_2608_07524_amd import _native as N
    rows, cols, ld = 37, 72, 200
    rng = np.random.default_rng(11)
    u, da = (to_device(torch, _bits(rng.standard_normal((rows, cols)))) for _ in range(2))
    wide = lambda: torch.full((rows, ld), 7.0, dtype=torch.bfloat16, device="cuda")
    uw, dw, o1, o2 = wide(), wide(), wide(), wide()
    uw[:, :cols], dw[:, :cols] = u, da
    kept = (u, None) if fmt == "bf16" else P.act8_pack(u, fmt)
    want = P.act8_gelu_bwd(*kept, da)
    d = N.Act8DescC(rows, cols, N.ACT_FORMATS[fmt], ld)
    src = (uw.data_ptr(), None) if fmt == "bf16" else tuple(t.data_ptr() for t in kept)
    N._check(N.load().dcp_act8_gelu_bwd(d, *src, dw.data_ptr(), o1.data_ptr(), o2.data_ptr(),
                                        torch.cuda.current_stream().cuda_stream))
    for got, ref in zip((o1, o2), want):
        assert torch.equal(got[:, :cols], ref) and bool((got[:, cols:] == 7.0).all())


def test_no_rows(torch, P):
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    codes, s = P.act8_pack(x)
    assert tuple(codes.shape) == (0, 64) and tuple(s.shape) == (0, 2)
    assert tuple(P.act8_unpack(codes, s).shape) == (0, 64)
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    r = P.gated_norm_fwd(x, x, g, g, g)
    b = P.gated_norm_bwd(x, x, x, x, r.rstd_f, r.rstd_out, g, g, g)
    assert not b.dpost.any() and not b.dgate.any() and not b.dpre.any()
    b = P.gated_norm_bwd(x, x, x, x, r.rstd_f, r.rstd_out, g, torch.ones(3, 64, dtype=torch.bfloat16, device="cuda"), g,
                         cu_seqlens=[0, 0, 0, 0])
    assert not b.dpost.any() and not b.dgate.any() and not b.dpre.any()


# ---------------------------------------------------------------------------
# joins

def _weights(torch, rng, h, n, post, gate, pre):
    made = {}
    if post:
        made["post"] = _bits(1 + 0.3 * rng.standard_normal(h))
    if gate != "none":
        made["gate"] = _bits(rng.standard_normal((n, h) if gate == "sequence" else h))
    if pre:
        made["pre"] = _bits(1 + 0.3 * rng.standard_normal(h))
    return {k: to_device(torch, v) for k, v in made.items()}, {k: I.bf16_to_f64(v) for k, v in made.items()}


def _case(torch, P, lengths, h, gate, post, pre, fmt, f32, alpha=1.0, extra=0, seed=0):
    """Forward and backward of one join against the oracle; `extra` rows lie behind
    the last sequence and have to stay as they are."""
    rng = np.random.default_rng(seed + h + len(lengths))
    cu = I.cu_from_lengths(lengths)
    T = int(cu[-1])
    rows = T + extra
    wt, w64 = _weights(torch, rng, h, len(lengths), post, gate, pre)
    xb, fb, gb = (_bits(rng.standard_normal((rows, h))) for _ in range(3))
    x, f, dout = (to_device(torch, b) for b in (xb, fb, gb))
    x64, f64, g64 = (I.bf16_to_f64(b)[:T] for b in (xb, fb, gb))
    per = cu if gate == "sequence" else None
    cu_t = None if per is None else torch.from_numpy(cu).cuda()
    keep = {} if fmt == "bf16" else dict(keep_f=fmt, **(dict(keep_out=fmt) if pre else {}))
    mark = lambda: torch.full((rows, h), 7.0, dtype=torch.bfloat16, device="cuda")
    kept = lambda t: bool((t[T:] == 7.0).all())
    r = P.gated_norm_fwd(x, f, cu_seqlens=cu_t, residual_scale=alpha, out=mark(), y=mark() if pre else None, **wt,
                         **keep)
    o = J.forward(x64, f64, cu=per, alpha=alpha, **w64)
    gates = J._gate_rows(w64.get("gate"), per, T)
    n = f64 if not post else f64 * o["rstd_f"][:, None] * w64["post"]
    mag = np.abs(alpha * x64) + np.abs(gates * n)
    _close("out", _f64(r.out)[:T], o["out"], mag, BF16)
    assert kept(r.out)
    if post:
        _close("rstd_f", r.rstd_f.cpu().numpy()[:T].astype(np.float64), o["rstd_f"], o["rstd_f"], 0)
    if pre:
        _close("rstd_out", r.rstd_out.cpu().numpy()[:T].astype(np.float64), o["rstd_out"], o["rstd_out"], 0)
        _close("y", _f64(r.y)[:T], o["y"], (mag * o["rstd_out"][:, None] * np.abs(w64["pre"])), BF16)
        assert kept(r.y)
    if fmt != "bf16":  # the checkpoints are those of f and of out as it was stored
        for got, of in ((r.f8, f), (r.out8, r.out)) if pre else ((r.f8, f),):
            c, s = P.act8_pack(of, fmt)
            assert torch.equal(got[0][:T].view(torch.uint8), c[:T].view(torch.uint8)) and torch.equal(got[1][:T], s[:T])
    # backward, from the values the kernels are given
    if fmt == "bf16":
        fk, ok, fv, ov = f, r.out, f64, _f64(r.out)[:T]
    else:
        fv, fk = _hold(torch, I.bf16_to_f64(fb), fmt)
        ov, ok = _hold(torch, _f64(r.out), fmt)
        fv, ov = fv[:T], ov[:T]
    dy = dy64 = None
    if pre:
        d = rng.standard_normal((rows, h)).astype(np.float32)
        dy = torch.from_numpy(d).cuda() if f32 else to_device(torch, _bits(d))
        dy64 = dy[:T].cpu().double().numpy()
    b = P.gated_norm_bwd(dout, dy, fk, ok if pre else None, r.rstd_f, r.rstd_out, cu_seqlens=cu_t, residual_scale=alpha,
                         want_y=pre, dx=mark(), df=mark(), y=mark() if pre else None, **wt)
    sc = lambda t: None if t is None else t.cpu().numpy()[:T].astype(np.float64)
    g, mag = J.backward(g64, dy64, fv, ov, sc(r.rstd_f), sc(r.rstd_out), cu=per, alpha=alpha, **w64)
    for n_ in ("dx", "df", "y"):
        if n_ in g:
            _close(n_, _f64(getattr(b, n_))[:T], g[n_], mag[n_], BF16)
            assert kept(getattr(b, n_)), n_
    for n_ in ("dpost", "dgate", "dpre"):
        t = getattr(b, n_)
        assert (t is None) == (n_ not in g)
        if t is not None:
            _close(n_, t.cpu().numpy().astype(np.float64), g[n_].reshape(t.shape), mag[n_].reshape(t.shape), 0)
    return r, b


# Widths of one lane, of part of a group, and at and beside the edges of every
# kernel's columns; lengths of none and one, sequences inside one team of rows,
# across two, and over more teams than a workgroup's parts (32 of 4 rows).
@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("h,lengths", [(8, [1]), (72, [0, 5, 0, 0, 1, 30, 0]), (256, [37, 64, 128, 200]),
                                       (288, [2, 90, 1]), (512, [7]), (520, [3, 4, 4, 1]), (1024, [9]), (1152, [1, 700, 16, 16, 33]),
                                       (1536, [2, 7]), (1544, [40, 1, 200]), (2048, [6]), (2304, [5, 150]),
                                       (2600, [30, 31]), (3080, [3, 0, 140]), (4096, [1, 21])])
def test_join_over_widths(torch, P, fmt, h, lengths):
    _case(torch, P, lengths, h, "sequence", True, True, fmt, False, extra=3)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("gate,post,pre", [("none", False, False), ("none", True, True), ("none", False, True),
                                           ("shared", True, True), ("shared", False, False), ("sequence", False, True),
                                           ("sequence", True, False), ("shared", False, True), ("none", True, False)])
def test_join_parts(torch, P, gate, post, pre, f32):
    for h, lengths in ((136, [50, 0, 61]), (2048, [33, 10])):
        _case(torch, P, lengths, h, gate, post, pre, "int8", f32, alpha=0.625, seed=int(f32))


# Many sequences: more than the workgroups that add their parts, more than one
# list of them holds, none with a row in its own team alone, and long ones in
# teams of more than 4 rows.
@pytest.mark.parametrize("h,lengths", [(64, [3] * 500), (8, [1] * 70000), (16, [13, 0, 5] * 900),
                                       (8, [20000, 7, 20001, 1, 30000])])
def test_join_many_rows(torch, P, h, lengths):
    _case(torch, P, lengths, h, "sequence", True, True, "int8", False, extra=1)


def test_join_of_more_than_2_31_elements(torch, P):
    """Offsets beyond 32 bits: the last rows equal a call on them alone."""
    rows, h, tail = 530_000, 4096, 300
    x = torch.empty(rows, h, dtype=torch.bfloat16, device="cuda").normal_()
    f = torch.empty(rows, h, dtype=torch.bfloat16, device="cuda").normal_()
    g = torch.full((h,), 1.25, dtype=torch.bfloat16, device="cuda")
    r = P.gated_norm_fwd(x, f, g, g, g, keep_f="int8", keep_out="int8")
    s = P.gated_norm_fwd(x[-tail:], f[-tail:], g, g, g, keep_f="int8", keep_out="int8")
    assert torch.equal(r.out[-tail:], s.out) and torch.equal(r.y[-tail:], s.y)
    for a, b in zip(r.f8 + r.out8, s.f8 + s.out8):
        assert torch.equal(a[-tail:], b)
    b = P.gated_norm_bwd(x, f, r.f8, r.out8, r.rstd_f, r.rstd_out, g, g, g, dx=x, df=f)
    x2 = torch.empty(tail, h, dtype=torch.bfloat16, device="cuda").normal_()
    assert bool(torch.isfinite(b.dpre).all()) and bool(torch.isfinite(b.dgate).all())
    c = P.gated_norm_bwd(x2, x2, s.f8, s.out8, s.rstd_f, s.rstd_out, g, g, g)
    x[-tail:], f[-tail:] = x2, x2
    d = P.gated_norm_bwd(x, f, r.f8, r.out8, r.rstd_f, r.rstd_out, g, g, g)
    assert torch.equal(d.dx[-tail:], c.dx) and torch.equal(d.df[-tail:], c.df)


def test_join_in_place_and_repeatable(torch, P):
    rng = np.random.default_rng(3)
    h, lengths = 1152, [40, 1, 90, 300]
    cu = torch.from_numpy(I.cu_from_lengths(lengths)).cuda()
    wt, _ = _weights(torch, rng, h, 4, True, "sequence", True)
    mk = lambda: to_device(torch, _bits(rng.standard_normal((431, h))))
    x, f, dout, dy = mk(), mk(), mk(), mk()
    a = P.gated_norm_fwd(x, f, cu_seqlens=cu, **wt)
    x2, f2 = x.clone(), f.clone()
    b = P.gated_norm_fwd(x2, f2, cu_seqlens=cu, out=x2, y=f2, **wt)
    assert torch.equal(a.out, b.out) and torch.equal(a.y, b.y)
    back = lambda **kw: P.gated_norm_bwd(kw.pop("dout", dout), kw.pop("dy", dy), f, a.out, a.rstd_f, a.rstd_out,
                                         cu_seqlens=cu, want_y=True, **wt, **kw)
    p, q = back(), back()
    d2, y2 = dout.clone(), dy.clone()
    r = back(dout=d2, dy=y2, dx=y2, df=d2)
    for n in ("dx", "df", "y", "dpost", "dgate", "dpre"):
        assert torch.equal(getattr(p, n), getattr(q, n)) and torch.equal(getattr(p, n), getattr(r, n)), n
    # dout None is a dout of zeros; dx may be left out
    z = back(dout=torch.zeros_like(dout))
    y = P.gated_norm_bwd(None, dy, f, a.out, a.rstd_f, a.rstd_out, cu_seqlens=cu, want_dx=False, **wt)
    assert torch.equal(z.df, y.df) and y.dx is None and torch.equal(z.dpre, y.dpre)
    f32 = P.gated_norm_bwd(None, dy.float(), f, a.out, a.rstd_f, a.rstd_out, cu_seqlens=cu, **wt)
    assert torch.equal(z.df, f32.df) and torch.equal(z.dx, f32.dx)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")  # (a workspace need not be cleared)
    own = back(workspace=ws)
    for n in ("dx", "df", "y", "dpost", "dgate", "dpre"):
        assert torch.equal(getattr(p, n), getattr(own, n)), n


def test_join_host_offsets_and_one_gate_row(torch, P):
    """Host offsets are the device's; one gate row is a gate for one sequence."""
    rng = np.random.default_rng(4)
    wt, _ = _weights(torch, rng, 128, 1, True, "sequence", True)
    x, f = (to_device(torch, _bits(rng.standard_normal((77, 128)))) for _ in range(2))
    a = P.gated_norm_fwd(x, f, cu_seqlens=[0, 77], **wt)
    b = P.gated_norm_fwd(x, f, **wt)
    assert torch.equal(a.out, b.out) and torch.equal(a.y, b.y)
    ga = P.gated_norm_bwd(x, f, f, a.out, a.rstd_f, a.rstd_out, cu_seqlens=[0, 77], **wt)
    gb = P.gated_norm_bwd(x, f, f, a.out, a.rstd_f, a.rstd_out, **wt)
    assert torch.equal(ga.df, gb.df) and torch.allclose(ga.dgate, gb.dgate, rtol=1e-5, atol=1e-4)


def test_join_nan_stays_in_its_row(torch, P):
    rng = np.random.default_rng(5)
    h = 1152
    g = torch.ones(h, dtype=torch.bfloat16, device="cuda")
    x, f = (to_device(torch, _bits(rng.standard_normal((40, h)))) for _ in range(2))
    clean = P.gated_norm_fwd(x, f, g, g, g, keep_f="int8")
    f[7, 100] = float("nan")
    f[9, 1151] = float("inf")
    r = P.gated_norm_fwd(x, f, g, g, g, keep_f="int8")
    others = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(r.out[others], clean.out[others]) and torch.equal(r.y[others], clean.y[others])
    assert bool(r.out[7].isnan().all()) and bool(r.y[9].isnan().any())
    held = P.act8_unpack(*r.f8)
    bad = held.isnan().nonzero().tolist()
    assert bad == [[7, c] for c in range(96, 128)] + [[9, c] for c in range(1120, 1152)]


def test_join_captured_and_replayed(torch, P):
    """Forward, GELU backward and join backward captured once, replayed on new
    inputs between eager calls, every replay against the eager result; two graphs
    with a workspace each replay in turn."""
    h, lengths = 256, [37, 64, 128, 200]
    rng = np.random.default_rng(6)
    cu = torch.from_numpy(I.cu_from_lengths(lengths)).cuda()
    wt, _ = _weights(torch, rng, h, 4, True, "sequence", True)
    st = [to_device(torch, _bits(rng.standard_normal((429, h)))) for _ in range(4)]

    def step(x, f, dout, dy):
        r = P.gated_norm_fwd(x, f, cu_seqlens=cu, keep_f="int8", keep_out="int8", **wt)
        du, a = P.act8_gelu_bwd(*r.f8, dout)
        b = P.gated_norm_bwd(du, dy, r.f8, r.out8, r.rstd_f, r.rstd_out, cu_seqlens=cu, want_y=True, **wt)
        return [r.out, r.y, a] + list(b)

    step(*st)
    graphs = []
    side = torch.cuda.Stream()
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            step(*st)
        side.synchronize()
        with torch.cuda.graph(g):
            outs = step(*st)
        graphs.append((g, outs))
    for i in range(4):
        for t in st:
            t.copy_(to_device(torch, _bits(rng.standard_normal((429, h)))))
        want = step(*st)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, outs in graphs:
            for a, b in zip(outs, want):
                assert torch.equal(a, b), i


def test_join_on_other_streams(torch, P):
    """Two calls at once on two streams, each with its own workspace."""
    rng = np.random.default_rng(8)
    h = 1152
    g = torch.ones(h, dtype=torch.bfloat16, device="cuda")
    data = [[to_device(torch, _bits(rng.standard_normal((4000, h)))) for _ in range(3)] for _ in range(2)]

    def step(x, f, d):
        r = P.gated_norm_fwd(x, f, g, g, g)
        return list(P.gated_norm_bwd(d, d, f, r.out, r.rstd_f, r.rstd_out, g, g, g, want_y=True))

    want = [step(*d) for d in data]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, d in zip(streams, data):
        with torch.cuda.stream(s):
            got.append(step(*d))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_join_keeps_either(torch, P, fmt):
    """A checkpoint of out alone, of f alone, and with no norm or gate at all: those of
    the matrices themselves."""
    rng = np.random.default_rng(10)
    for h in (72, 1152):
        x, f = (to_device(torch, _bits(rng.standard_normal((33, h)))) for _ in range(2))
        g = torch.ones(h, dtype=torch.bfloat16, device="cuda")
        for w in (dict(), dict(pre=g), dict(post=g, gate=g, pre=g)):
            for keep in (dict(keep_out=fmt), dict(keep_f=fmt)):
                r = P.gated_norm_fwd(x, f, residual_scale=0.5, **w, **keep)
                got, of = (r.out8, r.out) if "keep_out" in keep else (r.f8, f)
                assert (r.f8 is None) == ("keep_out" in keep) and (r.out8 is None) == ("keep_f" in keep)
                for a, b in zip(got, P.act8_pack(of, fmt)):
                    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
