"""dweight over many rows: a long sum, added in fp64."""
import pytest
import torch

import paper_2307_13592_amd as mgn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,cols", [(1_000_000, 128), (1_000_001, 33), (150_000, 1000), (100_000, 2049)])
def test_many_rows_add_up(n, cols):
    """Rows of ones with an eps that vanishes beside 1: u = 1 to a rounding, so
    each column's gradient is the sum of dy.  dy = 1 + 2^-19 has bits that a
    running fp32 sum past 32 drops, always downwards (2^-19 of each addend, 32
    half-steps); here each workgroup's partial and the result round once, and u
    and the product are off by a step and a half-step: 5 half-steps in all."""
    print(f"[rms] dweight of {n} x {cols}", flush=True)
    t = torch.ones(n, cols, device="cuda")
    dy = torch.full_like(t, 1 + 2.0 ** -19)
    dx, dw = torch.empty_like(t), torch.empty(cols, device="cuda")
    mgn.mgn_rms_norm_grad(t, None, dy, dx, dw, eps=2.0 ** -100)
    want = n * (1 + 2.0 ** -19)
    assert float((dw.double() - want).abs().max()) <= 5 * 2.0 ** -24 * want
