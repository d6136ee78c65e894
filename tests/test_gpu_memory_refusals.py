"""A refused call of a SelectiveMemory leaves it as it was: the convolution of a step
or window does not move `past` on, and a backward adds nothing to the gradients, if
the call that follows would be refused."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
from paper_2307_13592_amd.runner import SelectiveMemory

pytestmark = pytest.mark.gpu
T, ROWS, COLS, N, W = 6, 7, 12, 4, 3
REFUSED = (ValueError, mgn.MgnError)


def _memory(width=W):
    r = np.random.default_rng(width)
    t = lambda *s: torch.as_tensor(r.standard_normal(s).astype(np.float32)).cuda()
    m = SelectiveMemory(ROWS, COLS, N, width)
    for v in (m.conv_weight, m.conv_bias, m.dt_bias, m.state, m.past):
        v.copy_(t(*v.shape))
    return m, [t(T, ROWS, COLS), t(T, ROWS, COLS), t(T, ROWS, N), t(T, ROWS, N), t(T, ROWS, COLS)]


def _bad(m, x, dt, B, C, z):
    """Calls (x, dt, B, C, z) that the scan refuses, and the convolution does not."""
    yield "dt of other rows", (x, dt[..., 1:, :].contiguous(), B, C, z)
    yield "dt of another type", (x, dt.bfloat16(), B, C, z)
    yield "B of other states", (x, dt, B[..., 1:].contiguous(), C, z)
    yield "C on the host", (x, dt, B, C.cpu(), z)
    yield "z not contiguous", (x, dt, B, C, torch.stack([z, z], -1)[..., 0])
    yield "C of another type", (x, dt, B, C.double(), z)


@pytest.mark.parametrize("width", [1, 2, W])
def test_a_refused_step_or_window_leaves_the_memory(width):
    m, args = _memory(width)
    same, _ = _memory(width)
    state, past = m.state.clone(), m.past.clone()
    one = [a[0] for a in args]

    def refused(call, what):
        with pytest.raises(REFUSED):
            call()
        assert torch.equal(m.state, state) and torch.equal(m.past, past), what

    for what, bad in _bad(m, *one):
        refused(lambda: m.step(*bad), what)
    for what, bad in _bad(m, *args):
        refused(lambda: m.scan(*bad), what)
    A, m.A = m.A, m.A[1:].contiguous()
    refused(lambda: m.step(*one), "A of other columns")
    refused(lambda: m.scan(*args), "A of other columns")
    m.A = A
    y = m.step(*one)
    assert torch.equal(y, same.step(*one))
    state, past = m.state.clone(), m.past.clone()
    refused(lambda: m.step(*one[:4], y), "z: the last output, which the call overwrites")
    refused(lambda: m.step(one[0], m.state.view(-1)[:ROWS * COLS].view(ROWS, COLS), *one[2:]), "dt: a part of the state")
    window = [a[:1] for a in args]
    refused(lambda: m.scan(*window[:2], m.state.view(-1)[:ROWS * N].view(1, ROWS, N), *window[3:]), "B: a part of the state")
    # a right call afterwards is that of a memory which saw none of this
    assert torch.equal(m.scan(*args)[0], same.scan(*args)[0])
    assert torch.equal(m.state, same.state) and torch.equal(m.past, same.past)


def test_what_a_step_reads_is_not_what_its_convolution_moves():
    """past holds numbers of the step's own kind: given as a step's dt it is refused."""
    m, (x, dt, B, C, z) = _memory()
    state, past = m.state.clone(), m.past.clone()
    with pytest.raises(REFUSED):
        m.step(x[0], m.past[0], B[0], C[0], z[0])
    assert torch.equal(m.state, state) and torch.equal(m.past, past)


def test_a_refused_backward_adds_nothing():
    m, (x, dt, B, C, z) = _memory()
    y, kept = m.scan(x, dt, B, C, z)
    dy = torch.ones_like(y)
    m.grad(x, dt, B, C, kept, dy, z)
    before = {k: v.clone() for k, v in m.grads.items()}
    d_past = torch.ones(W - 1, ROWS, COLS, device="cuda")
    for kw in (dict(d_past=d_past[1:]), dict(d_past=d_past.bfloat16()), dict(d_past=d_past.cpu())):
        with pytest.raises(REFUSED):
            m.grad(x, dt, B, C, kept, dy, z, accumulate=True, **kw)
        assert all(torch.equal(m.grads[k], before[k]) for k in before)
    m.grad(x, dt, B, C, kept, dy, z, accumulate=True)
    for k, v in before.items():
        assert bool(((m.grads[k] - 2 * v).abs() <= 2.0 ** -22 * v.abs()).all()), k
