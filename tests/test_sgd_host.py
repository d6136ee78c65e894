"""Gradients that mgn_sgd_step would read as something else than they are, are refused
by their type: a bfloat16 one has half the bytes that the step reads (no GPU needed)."""
import pytest
import torch

import paper_2307_13592_amd as mgn


def test_gradients_of_another_type_or_length_are_refused():
    h = mgn.mgn_create(64, 1, 2)
    n = mgn.mgn_param_count(h)
    for dtype in (torch.bfloat16, torch.float16, torch.float64, torch.int32):
        with pytest.raises(ValueError, match="float32"):
            mgn.mgn_sgd_step(h, torch.zeros(n, dtype=dtype), 0.1)
    for m in (n - 1, n + 1, 0):
        with pytest.raises(ValueError, match="length"):
            mgn.mgn_sgd_step(h, torch.zeros(m), 0.1)
    with pytest.raises(ValueError, match="device"):
        mgn.mgn_sgd_step(h, torch.zeros(n), 0.1)
    for lr in (float("nan"), float("inf"), 1e39):
        with pytest.raises(mgn.MgnError):
            mgn.mgn_sgd_step(h, torch.zeros(n), lr)
    mgn.mgn_destroy(h)
