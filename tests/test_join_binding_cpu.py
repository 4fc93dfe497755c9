"""The binding of joins and checkpoints without a GPU: the stream that a call is given, and
the size of a join's workspace."""

import contextlib
import ctypes as C
import types

import pytest

import paper_2608_07524_amd as P
from paper_2608_07524_amd import _native as N


@pytest.mark.parametrize("raw", [True, False])
@pytest.mark.parametrize("current", [0, 1])
def test_calls_follow_the_current_stream_of_the_tensors_device(raw, current):
    """With and without the raw handles that some builds of torch offer."""
    entered = []

    @contextlib.contextmanager
    def device(d):
        entered.append(d.index)
        yield

    cuda = types.SimpleNamespace(current_device=lambda: current, device=device,
                                 current_stream=lambda d: types.SimpleNamespace(cuda_stream=100 + d.index))
    private = types.SimpleNamespace()
    if raw:
        private._cuda_getCurrentRawStream, private._cuda_getDevice = lambda i: 100 + i, lambda: current
    calls = []
    N._enqueue(types.SimpleNamespace(cuda=cuda, _C=private), types.SimpleNamespace(index=1),
               lambda *a: calls.append(a) or N.DCP_OK, 7)
    assert calls == [(7, 101)] and entered == ([] if current == 1 else [1])


@pytest.mark.parametrize("rows,hidden,n", [(0, 64, 0), (429, 256, 4), (12_001, 1152, 300), (5, 4096, 0)])
def test_workspace_size_of_a_join(rows, hidden, n):
    size = P.gated_norm_bwd_workspace_size(rows, hidden, n)
    d = N.GatedNormDescC(rows, hidden, n, 1 << 20 if n else None, 1.0, 0.0, N.ACT_BF16, 0, 0)
    want = C.c_size_t()
    assert P.load().dcp_gated_norm_bwd_workspace_size(d, want) == N.DCP_OK
    assert size == want.value and (size > 0) == (rows > 0)


@pytest.mark.parametrize("args", [(-1, 64), (8, 60), (8, 4104), (8, 64, -1)])
def test_workspace_size_refuses_what_the_call_would(args):
    with pytest.raises(P.DCPError):
        P.gated_norm_bwd_workspace_size(*args)
