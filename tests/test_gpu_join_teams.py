"""Joins whose teams of lanes own several rows: sequences that end and begin inside a team,
lie in one, and go on over few or many of them, against the definition in float64.  (At the
sizes of test_gpu_joins.py a team has one row, but for its cases of hidden 8.)

Tolerances, relative to the sums of magnitudes.  A row's sum passes 8 values a lane, 6 lane
steps and 8 wavefronts, 22 additions, of terms of up to three roundings; df joins three such
sums (the mean of d oh, and those of b t and b oh) and some eight further operations: fewer
than 2^6 roundings of 2^-24 along any path, 2^-18, and, in bf16, one of half a step, 2^-8 of
the value.  A weight's gradient adds such terms over a lane's rows (at most 128), a
workgroup's teams (at most 32) and the partial rows: columns 32 apart in eight running sums
(at most 2,560 / 256 = 10 each; along a sequence's teams at most 4,096 / 256 = 16), three
steps that join these and 32 parts.  Fewer than 128 + 32 + 16 + 3 + 32 = 211 roundings,
2^-16.2; with the terms' own 2^-18 below 2^-15."""

import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROUNDED, TERMS, SUMS = 2.0 ** -8, 2.0 ** -18, 2.0 ** -15
EPS = 1e-6


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


def _rows_of_a_team(rows, h, n_seqs):
    """From the workspace: two matrices of a partial row a workgroup, and two rows a team."""
    from paper_2608_07524_amd import _native as N
    size, one = C.c_size_t(), 4 * h
    d = N.GatedNormDescC(rows, h, n_seqs, 1 << 20 if n_seqs else None, 1.0, EPS, N.ACT_BF16, 0, 0)
    N._check(N.load().dcp_gated_norm_bwd_workspace_size(d, size))
    need = -(-h // 8)
    lanes = max(8, 1 << (need - 1).bit_length()) if need <= 64 else -(-need // 64) * 64
    teams = 256 // lanes if lanes <= 128 else 1
    blocks = size.value // (2 * one * (1 + (teams if n_seqs else 0)))
    return -(-rows // (blocks * teams))


def _lengths(rng, rows, kind):
    """Lengths that fill `rows`: all of one to a few rows, or short and long ones mixed;
    empty ones among them, first and last."""
    out, left = [0], rows
    while left:
        n = int(rng.choice([0, 1, 2, 3, 5, 17, 40] if kind == "short" else [0, 1, 3, 17, 51, 200, 700, 2000]))
        out.append(min(n, left))
        left -= out[-1]
    return out + [0, 0]


def _reference(torch, x, f, dout, dy, fk, ok, r, post, gate, pre, seq, n, alpha):
    """(forward, backward): values and magnitudes in float64; seq is each row's sequence (or
    None: one gate row), fk, ok, r what the backward is given."""
    d = lambda t: t.double()
    x, f, dout, dy, fk, ok, post, gate, pre = map(d, (x, f, dout, dy, fk, ok, post, gate, pre))
    rows = gate[seq] if seq is not None else gate.reshape(1, -1)
    mean = lambda t: t.mean(1, keepdim=True)
    fwd = {}
    rf = 1 / (mean(f * f) + EPS).sqrt()
    branch = rows * f * rf * post
    out, mag = alpha * x + branch, (alpha * x).abs() + branch.abs()
    ro = 1 / (mean(out * out) + EPS).sqrt()
    fwd["out"], fwd["y"] = (out, mag), (out * ro * pre, mag * ro * pre.abs())
    fwd["rstd_f"], fwd["rstd_out"] = (rf[:, 0], rf[:, 0]), (ro[:, 0], ro[:, 0])
    rf, ro = (d(t)[:, None] for t in r)
    oh, fh, g = ok * ro, fk * rf, pre * dy
    G = dout + ro * (g - oh * mean(g * oh))
    Gm = dout.abs() + ro * (g.abs() + oh.abs() * mean((g * oh).abs()))
    e, em = post * rows * G, (post * rows).abs() * Gm
    bwd = dict(dx=(alpha * G, abs(alpha) * Gm), y=(oh * pre, (oh * pre).abs()),
               df=(rf * (e - fh * mean(e * fh)), rf * (em + fh.abs() * mean(em * fh.abs()))),
               dpre=((dy * oh).sum(0), (dy * oh).abs().sum(0)),
               dpost=((rows * G * fh).sum(0), ((rows * fh).abs() * Gm).sum(0)))

    def gates(t):
        if seq is None:
            return t.sum(0).reshape(gate.shape)
        return torch.zeros(n, t.shape[1], dtype=torch.float64, device=t.device).index_add_(0, seq, t)

    bwd["dgate"] = gates(G * fh * post), gates(Gm * (fh * post).abs())
    return fwd, bwd


def _near(name, got, want, rel, abs_rel):
    (ref, mag), got = want, got.double()
    over = (got - ref).abs() - rel * ref.abs() - abs_rel * mag
    assert got.shape == ref.shape and bool((over <= 0).all()), (name, float(over.max()), int(over.argmax()))


def _check(torch, P, h, lengths, fmt, f32, kind="sequence", alpha=0.75, extra=5, least=2):
    rows = int(np.sum(lengths))
    gen = torch.Generator(device="cuda").manual_seed(rows + h)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)
    n = len(lengths) if kind == "sequence" else 0
    extra = extra if n else 0  # (rows behind the last sequence)
    team = _rows_of_a_team(rows + extra, h, n)
    print(f"h {h} rows {rows} sequences {n}: {team} rows a team", flush=True)
    assert team >= least
    x, f, dout = (rand(rows + extra, h) for _ in range(3))
    dy = rand(rows + extra, h)
    dy = dy.float() if f32 else dy
    post, pre, gate = 1 + 0.25 * rand(h), 1 + 0.25 * rand(h), rand(*((n, h) if n else (h,)))
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda() if n else None
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(lengths, device="cuda")) if n else None
    w = dict(post=post, gate=gate, pre=pre, cu_seqlens=cu, residual_scale=alpha)
    mark = lambda: torch.full((rows + extra, h), 7.0, dtype=torch.bfloat16, device="cuda")
    r = P.gated_norm_fwd(x, f, eps=EPS, out=mark(), y=mark(), **w)
    held = lambda t: (t, t) if fmt == "bf16" else (lambda k: (k, P.act8_unpack(*k)))(P.act8_pack(t, fmt))
    (fk, fv), (ok, ov) = held(f), held(r.out)
    b = P.gated_norm_bwd(dout, dy, fk, ok, r.rstd_f, r.rstd_out, want_y=True, dx=mark(), df=mark(), y=mark(), **w)
    own = slice(0, rows)
    fwd, bwd = _reference(torch, *(t[own] for t in (x, f, dout, dy, fv, ov)), (r.rstd_f[own], r.rstd_out[own]), post,
                          gate, pre, seq, n, alpha)
    for name in ("out", "y"):
        _near(name, getattr(r, name)[own], fwd[name], ROUNDED, TERMS)
    for name in ("rstd_f", "rstd_out"):
        _near(name, getattr(r, name)[own], fwd[name], 0, TERMS)
    for name in ("dx", "df", "y"):
        _near(name, getattr(b, name)[own], bwd[name], ROUNDED, TERMS)
    for name in ("dpost", "dpre", "dgate"):
        _near(name, getattr(b, name), bwd[name], 0, SUMS)
    if n:
        assert not b.dgate[0].any() and not b.dgate[-1].any()  # (empty sequences)
    for t in (r.out, r.y, b.dx, b.df, b.y):
        assert bool((t[rows:] == 7.0).all())


# A width for every number of lanes that a team has (8 to 512), rows for four to twenty rows
# a team, so that lengths of 1 to 40 rows end and begin anywhere in a team and 51 to 2,000 go
# on over a few or more than 32 teams.
@pytest.mark.parametrize("kind", ["short", "mixed"])
@pytest.mark.parametrize("h,rows,fmt,f32", [
    (64, 260_001, "int8", False), (72, 123_457, "bf16", True), (256, 61_443, "e4m3", False), (288, 40_961, "int8", True),
    (576, 20_011, "bf16", False), (1024, 12_289, "e4m3", True), (1152, 12_001, "int8", False),
    (1152, 23_003, "e4m3", True), (2048, 9_001, "bf16", True), (2304, 7_001, "int8", False), (2600, 6_001, "e4m3", False),
    (3080, 5_003, "bf16", False), (3584, 4_801, "int8", True), (4096, 5_003, "e4m3", True), (4096, 9_001, "bf16", False)])
def test_teams_of_several_rows(torch, P, h, rows, fmt, f32, kind):
    _check(torch, P, h, _lengths(np.random.default_rng(h + rows), rows, kind), fmt, f32, least=3)


@pytest.mark.parametrize("h,rows,fmt,f32", [(256, 50_000, "int8", True), (1152, 12_001, "bf16", False),
                                            (4096, 5_003, "int8", False)])
def test_one_gate_for_teams_of_several_rows(torch, P, h, rows, fmt, f32):
    _check(torch, P, h, [rows], fmt, f32, kind="shared", least=3)


# The longest sums: tens of rows in a lane, the most that one round of workgroups takes, and
# a second round.
@pytest.mark.parametrize("h,rows,least", [(512, 262_145, 50), (1152, 131_071, 100), (4096, 65_000, 120), (4096, 70_001, 60)])
def test_long_sums(torch, P, h, rows, least):
    rng = np.random.default_rng(h)
    lengths = [0, rows // 2 + 7, 1, rows // 3, 31, 64, 129]
    rest = rows - int(np.sum(lengths))
    _check(torch, P, h, lengths + [rest // 2, rest - rest // 2, 0, 0], str(rng.choice(["int8", "e4m3"])), False, least=least)


@pytest.mark.parametrize("h,rows", [(72, 123_457), (576, 20_011), (1152, 12_001), (4096, 5_003)])
def test_gradients_are_added_to(torch, P, h, rows):
    """The C call's accumulate = 1 adds to what is there: one sum, rounded (and, fused, one
    rounding of a product less): 2^-23 of the magnitudes.  Empty sequences' gradients stay."""
    from paper_2608_07524_amd import _native as N
    lengths = _lengths(np.random.default_rng(h), rows, "mixed")
    n = len(lengths)
    gen = torch.Generator(device="cuda").manual_seed(h)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, f, dout, dy = (rand(rows, h).to(torch.bfloat16) for _ in range(4))
    post, pre, gate = (rand(*s).to(torch.bfloat16) for s in ((h,), (h,), (n, h)))
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    r = P.gated_norm_fwd(x, f, post, gate, pre, cu)
    b = P.gated_norm_bwd(dout, dy, f, r.out, r.rstd_f, r.rstd_out, post, gate, pre, cu)
    there = [rand(h), rand(n, h), rand(h)]
    grads = [t.clone() for t in there]
    dx, df = torch.empty_like(x), torch.empty_like(x)
    d = N.GatedNormDescC(rows, h, n, cu.data_ptr(), 1.0, 0.0, N.ACT_BF16, 0, 1)
    size = C.c_size_t()
    N._check(N.load().dcp_gated_norm_bwd_workspace_size(d, size))
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    ptr = lambda *ts: [t.data_ptr() for t in ts]
    N._check(N.load().dcp_gated_norm_bwd(d, N.GatedNormPtrsC(*ptr(post, gate, pre)), *ptr(dout, dy),
                                         N.KeptC(f.data_ptr(), None), N.KeptC(r.out.data_ptr(), None),
                                         *ptr(r.rstd_f, r.rstd_out, dx, df), None, N.GatedNormPtrsC(*ptr(*grads)),
                                         ws.data_ptr(), size.value, torch.cuda.current_stream().cuda_stream))
    assert torch.equal(dx, b.dx) and torch.equal(df, b.df)
    for name, got, was, new in zip(("dpost", "dgate", "dpre"), grads, there, (b.dpost, b.dgate, b.dpre)):
        want = was.double() + new.double()
        assert bool(((got.double() - want).abs() <= 2.0 ** -23 * (was.abs() + new.abs()).double()).all()), name
    empty = torch.tensor([length == 0 for length in lengths], device="cuda")
    assert torch.equal(grads[1][empty], there[1][empty])
