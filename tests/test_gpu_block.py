"""GPU parity of the transformer block (dcp_block_fwd / dcp_block_bwd) against its
float64 oracle, with activations kept in bf16 and in 8 bits, and what holds
between its forms.

Tolerance: 2e-2 of the largest reference magnitude of each tensor, as for the
layer: the same bf16 products and intermediates, whose roundings (2^-8 relative) the
joins' norms carry on.  The backward's oracle is given the activations that the
stash holds.  (Holding its own would not do in 8 bits: an activation that the bf16
products moved by 2^-8 of itself falls on another code with a probability of 2^-8 over
the step, up to 2^-3 in e4m3, and is then a whole step away: in the mean square
sqrt(2^-8 2^-3) = 2 % of itself.)  What the stash holds is checked by itself: each
activation within the products' 2e-2 of the largest magnitude and the format's half
step."""

import math

import numpy as np
import pytest

from oracle import block as B
from paper_2608_07524_amd import inputs as I

from gpu_util import GRAD_TOL, to_bits, to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_07524_amd as P
    P.load()
    return t


def _setup(torch, lengths, H, D, causal, post, gates, fmt, alpha=1.0, seed=0, workspace=None):
    import paper_2608_07524_amd as P
    rng = np.random.default_rng(seed + 100 * H + len(lengths))
    h, cu = H * D, I.cu_from_lengths(lengths)
    W, Wd, G = {}, {}, {}
    for n, s in P.block_param_shapes(h, post, gates).items():
        v = 1.0 + 0.2 * rng.standard_normal(s) if n.startswith(("norm", "post")) else \
            rng.standard_normal(s) * (0.5 if "gate" in n else 1.0 / math.sqrt(s[0]))
        bits = I.bf16_bits(v.astype(np.float32))
        W[n], Wd[n] = I.bf16_to_f64(bits), to_device(torch, bits)
        G[n] = torch.zeros(s, dtype=torch.float32, device="cuda")
    xb, db = (I.bf16_bits(rng.standard_normal((int(cu[-1]), h)).astype(np.float32)) for _ in range(2))
    block = P.Block(Wd, G, cu, H, D, causal, None, 1e-6, workspace=workspace, stash_format=fmt, residual_scale=alpha)
    return block, cu, W, (I.bf16_to_f64(xb), I.bf16_to_f64(db)), (to_device(torch, xb), to_device(torch, db))


def _run(torch, block, x, dout, keep=True):
    for g in block.grads.values():
        g.zero_()
    out = block.fwd(x, keep=keep)
    dx = block.bwd(x, dout)
    torch.cuda.synchronize()
    return to_bits(out), to_bits(dx), {n: g.cpu().numpy().copy() for n, g in block.grads.items()}


def _stash(torch, block, fmt, H, branch):
    """What the stash holds, by dcp.h's layout."""
    raw, T, h, off = block.stash, block.T, block.hidden, 0

    def take(n, dtype, shape):
        nonlocal off
        t = raw[off:off + n].view(dtype).view(shape)
        off += -(-n // 256) * 256
        return t

    import paper_2608_07524_amd as P
    kept = {}
    for name in ("q", "k", "v", "o") + (("f1",) if branch else ()) + ("h",) + (("f2",) if branch else ()) + ("u",):
        cols = 4 * h if name == "u" else h
        if fmt == "bf16" or name == "o":
            t = take(2 * T * cols, torch.bfloat16, (T, cols))
        else:
            codes = take(T * cols, torch.int8 if fmt == "int8" else torch.float8_e4m3fn, (T, cols))
            t = P.act8_unpack(codes.clone(), take(T * -(-cols // 32), torch.uint8, (T, -(-cols // 32))).clone())
        kept[name] = t.double().cpu().numpy()
    kept["lse"] = take(4 * H * T, torch.float32, (H, T)).double().cpu().numpy()
    for name in ("rstd_f1", "rstd_h", "rstd_f2"):
        kept[name] = take(4 * T, torch.float32, (T,)).double().cpu().numpy()
    assert off == block.stash_bytes
    return kept


def _errors(torch, block, cu, W, host, dev, H, D, causal, fmt, alpha):
    for g in block.grads.values():
        g.zero_()
    out = block.fwd(dev[0])
    held = _stash(torch, block, fmt, H, "post1" in W or "gate1" in W)
    dx = block.bwd(*dev)
    torch.cuda.synchronize()
    args = (cu, H, D, 1.0 / math.sqrt(D), causal, 1e-6, alpha)
    ref, kept = B.forward(host[0], W, *args)
    for n in ("q", "k", "v", "o", "f1", "h", "f2", "u"):
        if n in held:
            top = np.max(np.abs(kept[n]))
            # (the half step of a group is at most that of the largest magnitude: 1 / 127 of
            # it, or 2^-4; with what the products moved, 1.02 of it)
            half = {"bf16": 0.0, "int8": 1.02 / 127, "e4m3": 1.02 / 16}["bf16" if n == "o" else fmt] * top
            assert np.max(np.abs(held[n] - kept[n])) <= GRAD_TOL * top + half, n
    for n in ("f1", "f2"):
        held.setdefault(n, None)
    if "post1" not in W:
        held["rstd_f1"] = held["rstd_f2"] = None
    rdx, rg = B.backward(host[1], host[0], W, held, *args)
    rel = lambda a, b: float(np.max(np.abs(a - b)) / np.max(np.abs(b)))
    errs = {"out": rel(I.bf16_to_f64(to_bits(out)), ref), "dx": rel(I.bf16_to_f64(to_bits(dx)), rdx)}
    got = {n: g.double().cpu().numpy() for n, g in block.grads.items()}
    # (one token, whose query and key have no gradient, is given what v's rounding leaves of
    # dO . v - dO . o: the same on both sides)
    errs.update({n: rel(got[n], rg[n]) for n in rg})
    print(f"block {fmt} H={H} D={D} T={len(dx)}: " + " ".join(f"{k} {v:.1e}" for k, v in errs.items()), flush=True)
    return errs


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("post,gate,causal,alpha", [(True, "sequence", False, 1.0), (True, "shared", True, 0.625),
                                                    (False, "sequence", True, 1.0), (True, "none", False, 0.625),
                                                    (False, "none", True, 1.0), (False, "none", False, 0.625)])
def test_block_matches_oracle(torch, fmt, post, gate, causal, alpha):
    lengths, H, D = [300, 45, 0, 17, 700, 1, 130], 2, 64
    gates = {"none": 0, "shared": 1, "sequence": len(lengths)}[gate]
    block, cu, W, host, dev = _setup(torch, lengths, H, D, causal, post, gates, fmt, alpha)
    errs = _errors(torch, block, cu, W, host, dev, H, D, causal, fmt, alpha)
    assert max(errs.values()) <= GRAD_TOL, errs


# Widths with a short last group of columns, of the video model's heads, and wide;
# token counts on both sides of those from which the products change kernels.
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,D,lengths", [(1, 72, [1]), (3, 72, [513]), (1, 64, [512, 3]), (4, 72, [2047, 66]),
                                         (16, 72, [300, 277]), (16, 128, [33]), (1, 72, [70] * 88)])
def test_block_sizes_and_products(torch, fmt, H, D, lengths):
    block, cu, W, host, dev = _setup(torch, lengths, H, D, True, True, len(lengths), fmt)
    errs = _errors(torch, block, cu, W, host, dev, H, D, True, fmt, 1.0)
    assert max(errs.values()) <= GRAD_TOL, errs


@pytest.mark.parametrize("post,gates,alpha", [(True, 4, 1.0), (False, 0, 1.0), (False, 0, 0.5)])
def test_forms_agree(torch, post, gates, alpha):
    """The output does not depend on the stash; a recomputing backward has the bits of
    one from a bf16 stash, whatever the format; every form repeats its bits."""
    lengths, H, D = [200, 37, 513, 9], 4, 72
    results = {}
    for fmt in ("bf16", "int8", "e4m3"):
        block, _, _, _, dev = _setup(torch, lengths, H, D, False, post, gates, fmt, alpha, seed=5)
        results[fmt] = _run(torch, block, *dev)
        again = _run(torch, block, *dev)
        results[fmt, "recomputed"] = _run(torch, block, *dev, keep=False)
        assert np.array_equal(results[fmt][1], again[1])
        assert all(np.array_equal(results[fmt][2][n], again[2][n]) for n in again[2])
    base = results["bf16"]
    for key, r in results.items():
        assert np.array_equal(base[0], r[0]), key
        if key == "bf16" or isinstance(key, tuple):
            assert np.array_equal(base[1], r[1]), key
            assert all(np.array_equal(base[2][n], r[2][n]) for n in base[2]), key
    assert not np.array_equal(base[1], results["int8"][1])


def test_gradients_add_up_and_streams(torch):
    """A second backward adds to the gradients, and a block follows the current stream."""
    lengths = [64, 31, 100]
    block, _, _, _, (x, dout) = _setup(torch, lengths, 2, 64, True, True, 3, "int8")
    _, dx, once = _run(torch, block, x, dout)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block.fwd(x)
        dx2 = block.bwd(x, dout)
    torch.cuda.synchronize()
    assert np.array_equal(to_bits(dx2), dx)
    for n, g in block.grads.items():
        # (twice a value is exact; sums that add to what is there round once more: 2^-24 of
        # the partial sums' magnitudes, which for these few rows stay below 2^6 of the largest)
        assert np.max(np.abs(g.cpu().numpy() - 2 * once[n])) <= 2.0 ** -18 * max(np.max(np.abs(once[n])), 1e-30), n


def test_stash_buffer_and_shared_workspace(torch):
    """Two blocks on one workspace, each with a stash of its own, run forward and
    backward in turn as a stack does: the bits of each alone."""
    lengths = [100, 20, 300]
    a, _, _, _, (x, dout) = _setup(torch, lengths, 2, 64, False, True, 3, "int8", seed=1)
    b, _, _, _, _ = _setup(torch, lengths, 2, 64, False, True, 3, "int8", seed=2, workspace=a.ws)
    alone_a = _run(torch, a, x, dout)
    y = a.fwd(x)
    alone_b = _run(torch, b, y, dout)
    for g in list(a.grads.values()) + list(b.grads.values()):
        g.zero_()
    stash = [torch.full((a.stash_bytes + 512,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    y = a.fwd(x, stash=stash[0][256:256 + a.stash_bytes])
    b.fwd(y, stash=stash[1][256:256 + a.stash_bytes])
    dy = b.bwd(y, dout)
    a.bwd(x, dout)
    torch.cuda.synchronize()
    assert np.array_equal(to_bits(dy), alone_b[1])
    for block, alone in ((a, alone_a), (b, alone_b)):
        for n, g in block.grads.items():
            assert np.array_equal(g.cpu().numpy(), alone[2][n]), n
    for t in stash:  # nothing outside the stash was written
        assert bool((t[:256] == 255).all()) and bool((t[256 + a.stash_bytes:] == 255).all())
    with pytest.raises(ValueError, match="stash"):
        a.fwd(x, stash=stash[0][:a.stash_bytes - 1])


def test_no_tokens(torch):
    block, _, _, _, (x, dout) = _setup(torch, [0, 0], 2, 64, False, True, 2, "int8")
    assert tuple(block.fwd(x).shape) == (0, 128) and tuple(block.bwd(x, dout).shape) == (0, 128)


def test_join_by_join(torch):
    """The block's halves made of the public operators, as a program that builds its
    own block would call them: attention and its join, kept in 8 bits, forward and
    backward, against the oracle's join on the same inputs."""
    import paper_2608_07524_amd as P
    from oracle import attention as A
    from oracle import join as J
    rng = np.random.default_rng(9)
    H, D, lengths = 4, 64, [37, 64, 128, 200]
    h, cu = H * D, I.cu_from_lengths(lengths)
    T = int(cu[-1])
    bits = lambda *s: I.bf16_bits(rng.standard_normal(s).astype(np.float32))
    q, k, v, xb, gb, db = (bits(T, h) for _ in range(6))
    wb = {n: bits(*s) for n, s in (("post", (h,)), ("gate", (4, h)), ("pre", (h,)))}
    dev = lambda b: to_device(torch, b)
    w = {n: dev(b) for n, b in wb.items()}
    heads = lambda b: dev(b).view(T, H, D)
    o, lse = P.varlen_attn_fwd(heads(q), heads(k), heads(v), cu)
    cu_t = torch.from_numpy(cu).cuda()
    r = P.gated_norm_fwd(dev(xb), o.view(T, h), cu_seqlens=cu_t, keep_f="int8", keep_out="int8", **w)
    g = P.gated_norm_bwd(dev(gb), dev(db), r.f8, r.out8, r.rstd_f, r.rstd_out, cu_seqlens=cu_t, want_y=True, **w)
    dq, dk, dv = P.varlen_attn_bwd(g.df.view(T, H, D), o, lse, heads(q), heads(k), heads(v), cu)
    f64 = lambda b: I.bf16_to_f64(b)
    w64 = {n: f64(b) for n, b in wb.items()}
    q64, k64, v64 = (f64(b).reshape(T, H, D) for b in (q, k, v))
    ro, _ = A.attention_forward(q64, k64, v64, cu, 1 / 8, False)
    j = J.forward(f64(xb), ro.reshape(T, h), cu=cu, **w64)
    held = lambda kept: f64(to_bits(P.act8_unpack(*kept)))
    jg, _ = J.backward(f64(gb), f64(db), held(r.f8), held(r.out8), j["rstd_f"], j["rstd_out"], cu=cu, **w64)
    refs = A.attention_backward(jg["df"].reshape(T, H, D), q64, k64, v64, cu, 1 / 8, False)
    rel = lambda t, ref: float(np.max(np.abs(t.double().cpu().numpy().reshape(ref.shape) - ref)) / np.max(np.abs(ref)))
    errs = {n: rel(getattr(r, n), j[n]) for n in ("out", "y")}
    errs.update({n: rel(getattr(g, n), jg[n]) for n in ("dx", "df", "y", "dpost", "dgate", "dpre")})
    errs.update({n: rel(t, ref) for n, t, ref in zip(("dq", "dk", "dv"), (dq, dk, dv), refs)})
    print("join by join: " + " ".join(f"{n} {e:.1e}" for n, e in errs.items()), flush=True)
    assert max(errs.values()) <= GRAD_TOL, errs


@pytest.mark.parametrize("gated", [False, True])
def test_stack_of_blocks(torch, gated):
    """Three blocks through the executor: the output is the bf16 stack's whatever is
    kept, a recompute pattern's gradients are those of the layers it keeps, and the
    dual-layer row's m is the stash."""
    from paper_2608_07524_amd import model as M
    cu = [0, 150, 170, 400]
    kind = dict(post_norm=gated, gates=3 if gated else 0)
    results = {}
    for fmt in ("bf16", "int8"):
        st = M.Stack(3, cu, 2, 64, causal=True, seed=4, stash_format=fmt, **kind)
        for flags in ([0, 0, 0], [1, 0, 0], [1, 1, 1]):
            for layer in st.layers:
                for g in layer.grads.values():
                    g.zero_()
            st.step(flags)
            torch.cuda.synchronize()
            grads = [layer.grads[n].cpu().numpy().copy() for layer in st.layers for n in layer.grads]
            results[fmt, sum(flags)] = to_bits(st.xs[-1]), to_bits(st.dys[0]), grads
    base = results["bf16", 0]
    for key, r in results.items():
        assert np.array_equal(r[0], base[0]), key
        if key[0] == "bf16" or key[1] == 3:
            assert np.array_equal(r[1], base[1]) and all(np.array_equal(a, b) for a, b in zip(r[2], base[2])), key
    kind["gates"] = min(kind["gates"], 1)  # (a profile's length is one sequence)
    rows = {fmt: M.profile_rows([256], 2, 64, True, reps=2, warmup=1, stash_format=fmt, **kind)[0] for fmt in
            ("bf16", "int8")}
    assert rows["int8"].m_bytes < 0.6 * rows["bf16"].m_bytes and rows["int8"].t_f_ns > 0


def test_eight_bit_gradients_are_near(torch):
    """Through a stack of blocks the gradients from 8-bit stashes stay near those from
    bf16, in the first block as in the last: relative errors of the order of the formats'
    own (0.8 % of the standard deviation, 2.7 %), at most four times that.  (A query's or
    key's gradient multiplies three held matrices, its noise adds in quadrature, sqrt(3) of
    one; the weights' e^(logit) adds as much again, and inputs and dY1 carry the later
    blocks' errors.  With o in 8 bits dWq of the last block is off by 7 and 23 %.)"""
    from paper_2608_07524_amd import model as M
    res = {}
    for fmt in ("bf16", "int8", "e4m3"):
        st = M.Stack(4, [0, 1024, 2048, 4096], 16, 72, False, seed=3, stash_format=fmt, post_norm=True, gates=3)
        st.step([0] * 4)
        torch.cuda.synchronize()
        res[fmt] = [st.dys[0].float()] + [layer.grads[n].clone() for layer in st.layers for n in layer.grads]
    for fmt, own in (("int8", 0.0083), ("e4m3", 0.027)):
        errs = [float((a - b).norm() / b.norm()) for a, b in zip(res[fmt], res["bf16"])]
        print(f"{fmt}: " + " ".join(f"{e:.4f}" for e in errs), flush=True)
        assert max(errs) <= 4 * own


def test_wide_block_of_many_tokens(torch):
    """Hidden 4,096 from 12,288 tokens on: the library's weight gradients, and no fused
    products; the sum of the gradients of the batch's halves."""
    import paper_2608_07524_amd as P
    H, D, T = 32, 128, 12288
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    W = {n: (rand(*s) / (math.sqrt(s[0]) if n.startswith("w") else 1.0)).to(torch.bfloat16)
         for n, s in P.block_param_shapes(H * D, True, 1).items()}
    x, dout = (rand(T, H * D).to(torch.bfloat16) for _ in range(2))

    def grads(rows):
        g = {n: torch.zeros(w.shape, dtype=torch.float32, device="cuda") for n, w in W.items()}
        for lo in range(0, T, rows):
            block = P.Block(W, g, np.arange(0, rows + 1, 512), H, D, True, None, 1e-6, stash_format="int8")
            block.fwd(x[lo:lo + rows])
            block.bwd(x[lo:lo + rows], dout[lo:lo + rows])
            torch.cuda.synchronize()
        return g

    whole, halves = grads(T), grads(T // 2)
    errs = {n: float((whole[n] - halves[n]).abs().max() / halves[n].abs().max()) for n in W}
    assert max(errs.values()) <= GRAD_TOL, errs
