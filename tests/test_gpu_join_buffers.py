"""Buffers that a call may share: outputs in the places of inputs, and slices of one wider
matrix beside each other, give the bits of buffers of their own."""

import numpy as np
import pytest

from paper_2608_07524_amd import inputs as I

from gpu_util import to_device

pytestmark = pytest.mark.gpu


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


def _rand(torch, rng, *shape):
    return to_device(torch, I.bf16_bits(rng.standard_normal(shape).astype(np.float32)))


@pytest.mark.parametrize("h", [72, 1152, 4096])
def test_join_backward_in_the_kept_activations(torch, P, h):
    """dx, df and y over f, out, dout and dy as kept in bf16, in every assignment."""
    rng = np.random.default_rng(h)
    rows, g = 301, _rand(torch, rng, h)
    x, f, dout, dy = (_rand(torch, rng, rows, h) for _ in range(4))
    r = P.gated_norm_fwd(x, f, g, g, g)
    back = lambda t, **kw: P.gated_norm_bwd(t["dout"], t["dy"], t["f"], t["out"], r.rstd_f, r.rstd_out, g, g, g,
                                            want_y=True, **kw)
    data = dict(dout=dout, dy=dy, f=f, out=r.out)
    want = back(data)
    names = list(data)
    for i in range(4):
        t = {n: v.clone() for n, v in data.items()}
        got = back(t, dx=t[names[i]], df=t[names[(i + 1) % 4]], y=t[names[(i + 2) % 4]])
        for a, b in zip(got, want):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_gelu_backward_between_slices_of_one_matrix(torch, P, fmt):
    """da, du, a (and a bf16 u) as neighbouring column slices of one matrix."""
    from paper_2608_07524_amd import _native as N
    rng = np.random.default_rng(1)
    rows, cols = 37, 72
    u, da = _rand(torch, rng, rows, cols), _rand(torch, rng, rows, cols)
    kept = (u, None) if fmt == "bf16" else P.act8_pack(u, fmt)
    want = P.act8_gelu_bwd(*kept, da)
    wide = torch.full((rows, 4 * cols), 7.0, dtype=torch.bfloat16, device="cuda")
    part = [wide[:, i * cols:(i + 1) * cols] for i in range(4)]
    part[0].copy_(da)
    part[3].copy_(u)
    src = (part[3].data_ptr(), None) if fmt == "bf16" else tuple(t.data_ptr() for t in kept)
    d = N.Act8DescC(rows, cols, N.ACT_FORMATS[fmt], 4 * cols)
    N._check(N.load().dcp_act8_gelu_bwd(d, *src, part[0].data_ptr(), part[1].data_ptr(), part[2].data_ptr(),
                                        torch.cuda.current_stream().cuda_stream))
    assert torch.equal(part[1], want[0]) and torch.equal(part[2], want[1])
    assert torch.equal(part[0], da) and torch.equal(part[3], u)


def test_checkpoints_beside_each_other(torch, P):
    """A checkpoint in memory that ends where its matrix begins, and of one slice beside
    another's: no byte is shared."""
    rng = np.random.default_rng(2)
    rows, cols = 16, 64
    x = _rand(torch, rng, rows, cols)
    raw = torch.zeros(rows * cols * 3 + rows * 2, dtype=torch.uint8, device="cuda")
    codes, rest = raw[:rows * cols].view(torch.int8).view(rows, cols), raw[rows * cols:]
    inside = rest[:2 * rows * cols].view(torch.bfloat16).view(rows, cols)
    scales = rest[2 * rows * cols:].view(rows, 2)
    inside.copy_(x)
    got = P.act8_pack(inside, "int8", codes, scales)
    want = P.act8_pack(x, "int8")
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(inside, x)
    wide = torch.cat([x, x], 1)
    back = P.act8_unpack(*want, out=wide[:, cols:])
    assert torch.equal(back, P.act8_unpack(*want)) and torch.equal(wide[:, :cols], x)


def test_workspace_of_the_stated_size(torch, P):
    """gated_norm_bwd_workspace_size is enough, nothing behind it is written, and a byte less
    is refused."""
    rng = np.random.default_rng(3)
    rows, h, cu = 5000, 1152, [0, 7, 7, 2000, 2003, 4990]
    g, gate = _rand(torch, rng, h), _rand(torch, rng, len(cu) - 1, h)
    x, f, dout = (_rand(torch, rng, rows, h) for _ in range(3))
    r = P.gated_norm_fwd(x, f, g, gate, g, cu)
    back = lambda **kw: P.gated_norm_bwd(dout, dout, f, r.out, r.rstd_f, r.rstd_out, g, gate, g, cu, **kw)
    size = P.gated_norm_bwd_workspace_size(rows, h, len(cu) - 1)
    room = torch.full((size + 256,), 255, dtype=torch.uint8, device="cuda")
    got, want = back(workspace=room[:size]), back()
    for name in ("dpost", "dgate", "dpre"):
        assert torch.equal(getattr(got, name), getattr(want, name)), name
    assert bool((room[size:] == 255).all())
    with pytest.raises(P.DCPError, match="workspace"):
        back(workspace=room[:size - 1])
