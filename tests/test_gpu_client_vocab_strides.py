"""The losses over a vocabulary through the C ABI: the row stride of a matrix of
one row may be anything, as elsewhere in include/fasgd_client.h."""
import ctypes
import math

import pytest
import torch

from paper_1601_04033_amd import client
from test_gpu_client_vocab import DTYPES, Case, reference, workspace
from vocab_ways import way

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m, d, V, form", [(2 ** 19 + 17, 8, 1, "tiles"), (40, 24, 1, "direct"), (1, 24, 40, "direct"),
                                           (1, 8, 2 ** 26 + 1, "tiles")])
def test_strides_of_a_single_row(dtype, m, d, V, form):
    assert way(m, d, V, DTYPES[dtype]) == form
    lib = client._library()
    c = Case(dtype, m, d, V) if V < 1000 else None
    if c is None:       # a vocabulary too large for the reference: the same call with strides that are right
        g = torch.Generator(device="cuda").manual_seed(3)
        c = Case(dtype, m, d, 2)
        c.w = torch.randn(V, d, device="cuda", generator=g).to(c.dt)
    kind = client._dtype(c.x, "x")
    stream = torch.cuda.current_stream().cuda_stream
    new = lambda *s, **k: torch.full(s, math.nan, device="cuda", **k)
    results = []
    for ld in (d, 0, -8, 3):
        head = client.client_vocab_head(m, d, V, kind, 1.0, c.x.data_ptr(), ld if m == 1 else d, c.w.data_ptr(),
                                        ld if V == 1 else d)
        loss, lse, picked, dx, dw = new(m), new(m), new(m), new(m, d, dtype=c.dt), new(V, d)
        ws = workspace(c, False)
        assert lib.client_vocab_loss_forward(ctypes.byref(head), c.index.data_ptr(), 0.0, 0.1, loss.data_ptr(),
                                             lse.data_ptr(), picked.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
        ws = workspace(c, True)
        assert lib.client_vocab_loss_backward(ctypes.byref(head), c.index.data_ptr(), 0.0, 0.1, lse.data_ptr(),
                                              picked.data_ptr(), c.dloss.data_ptr(), 1.0, dx.data_ptr(),
                                              ld if m == 1 else d, dw.data_ptr(), ld if V == 1 else d, 0, 0,
                                              ws.data_ptr(), ws.numel(), stream) == 0
        results.append((loss, lse, picked, dx, dw))
        del ws
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
    if V < 1000:
        ref = reference(c, z_loss=0.1)
        for name, got in zip(("loss", "lse", "picked", "dx", "dw"), results[0]):
            ref.check(name, got)
