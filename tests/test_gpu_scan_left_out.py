"""Selective scan and convolution: a parameter that is left out stands for zeros, and
its gradient, if it is asked for, is the gradient there."""
import pytest
import torch

import paper_2307_13592_amd as mgn
from test_gpu_selective_scan import _args, _backward, _case, _forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,n", [(1, 3, 5, 2), (20, 33, 64, 16), (9, 5, 77, 33), (300, 1, 20, 5)])
@pytest.mark.parametrize("gate", [False, True])
def test_scan_without_some(T, rows, cols, n, dtype, gate):
    zeros = torch.zeros(cols, device="cuda")
    for left in (("D",), ("bias",), ("h0",), ("D", "bias", "h0", "dh_last")):
        c = _case(T, rows, cols, n, dtype, gate=gate, starts=0.1, seed=21)
        there, none = dict(c), dict(c)
        for k in left:
            there[k] = torch.zeros_like(c[k])
            none[k] = None
        y, last, marks = _forward(there)
        want = _backward(there, marks)
        y0, last0, marks0 = _forward(none)
        assert torch.equal(y, y0) and torch.equal(last, last0) and torch.equal(marks, marks0)
        e = torch.empty_like
        got = dict(dx=e(y), ddt=e(y), dA=e(c["A"]), dB=e(c["B"]), dC=e(c["C"]), dz=e(y) if gate else None, dD=torch.full_like(zeros, 7.0),
                   d_bias=torch.full_like(zeros, 7.0), dh0=e(last))
        mgn.mgn_selective_scan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], marks0, c["dy"], dh_last=none["dh_last"], **got, **_args(none))
        for k, v in want.items():
            assert torch.equal(got[k], v), (left, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,rows,cols,W", [(1, 3, 5, 4), (2, 7, 64, 8), (20, 33, 64, 4), (300, 1, 21, 3)])
@pytest.mark.parametrize("silu", [False, True])
def test_convolution_without_some(T, rows, cols, W, dtype, silu):
    t = lambda *s: torch.randn(*s, device="cuda")
    x, dy, w = t(T, rows, cols).to(dtype), t(T, rows, cols).to(dtype), t(cols, W)
    starts = (torch.rand(T, device="cuda") < 0.1).to(torch.uint8)
    runs = []
    for bias, past, d_out in ((torch.zeros(cols, device="cuda"), torch.zeros(W - 1, rows, cols, dtype=dtype, device="cuda"),
                               torch.zeros(W - 1, rows, cols, device="cuda")), (None, None, None)):
        y, left = torch.empty_like(x), torch.empty(W - 1, rows, cols, dtype=dtype, device="cuda")
        mgn.mgn_causal_conv(x, w, y, bias=bias, past=past, past_out=left, starts=starts, silu=silu)
        g = [torch.empty_like(x), torch.empty_like(w), torch.empty(cols, device="cuda"), torch.empty(W - 1, rows, cols, device="cuda")]
        mgn.mgn_causal_conv_grad(x, w, dy, g[0], g[1], g[2], bias=bias, past=past, d_past=g[3], d_past_out=d_out, starts=starts, silu=silu)
        runs.append([y, left] + g)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_without_some(dtype):
    rows, cols = 301, 100
    x, dy = torch.randn(rows, cols, device="cuda").to(dtype), torch.randn(rows, cols, device="cuda").to(dtype)
    runs = []
    for w, b in ((torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")), (None, None)):
        y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        mgn.mgn_layer_norm(x, w, b, y)
        mgn.mgn_layer_norm_grad(x, w, dy, dx, dw, db)
        runs.append([y, dx, dw, db])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
