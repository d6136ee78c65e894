"""Norms and clipping at the ends of fp32's range, and over several tables of tensors.
The norm is rounded once, the factor once, its product with a value once and the
result once to its type; below fp32's normal numbers a step is 2^-149."""
import numpy as np
import pytest
import torch

import memory_ref as ref
import paper_2307_13592_amd as mgn

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -149


def _clip(gs, most, given=None):
    outs = [torch.full_like(g, 9.0) for g in gs]
    norm = torch.empty(1, device="cuda") if given is None else torch.tensor([given], dtype=torch.float32, device="cuda")
    mgn.mgn_grad_clip(mgn.mgn_grad_list(gs, outs), most, norm, given=given is not None)
    return outs, float(norm)


def _near(out, want):
    lim = 4 * ref.U * np.abs(want) + (ref.half(out.dtype) - ref.U) * np.abs(want) * 1.01
    lim += STEP if out.dtype == torch.float32 else 2.0 ** -133  # (bf16's step there)
    err = np.abs(ref.f64(out) - want)
    assert bool((err <= lim).all()), float((err / lim).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale,over", [(1e-30, 3.0), (1e-20, 1e3), (1e18, 1e3), (1e30, 1e38), (1e30, 1e39), (1e34, 3e41), (1e30, 1e45), (1e34, 1e60),
                                        (1e34, 1e75), (1e-18, 1e20)])
def test_factors_of_any_size(scale, over, dtype):
    """max_norm / norm down to fp32's subnormal numbers and far below them."""
    r = np.random.default_rng(5)
    gs = [torch.as_tensor((scale * r.standard_normal(m)).astype(np.float32)).cuda().to(dtype) for m in (1000, 77, 8195)]
    want = float(np.sqrt(sum(float((g.double() ** 2).sum()) for g in gs)))
    most = float(np.float32(want / over))
    for given in (None, want):
        outs, norm = _clip(gs, most, given)
        assert abs(norm - want) <= 1.01 * ref.U * want
        for g, o in zip(gs, outs):
            _near(o, ref.f64(g) * (most / want))
    kept = [g.clone() for g in gs]
    assert all(torch.equal(a, b) for a, b in zip(_clip(gs, 3e38)[0], kept))


@pytest.mark.parametrize("count,length,dtype", [(3600, 8193, torch.float32), (300, 500_003, torch.bfloat16), (300, 400_003, torch.bfloat16)])
def test_several_tables(count, length, dtype):
    """More tensors than one launch takes, with more partials (the first) or more tiles
    than a scaling workgroup adds or takes itself, and with fewer."""
    flat = torch.empty(count * length, dtype=dtype, device="cuda")
    for part in flat.split(1 << 27):
        part.normal_()
    out = torch.empty_like(flat)
    total = sum(float((p.double() ** 2).sum()) for p in flat.split(1 << 25))
    want = total ** 0.5
    norm = torch.empty(1, device="cuda")
    lst = mgn.mgn_grad_list(flat.split(length), out.split(length))
    mgn.mgn_grad_norm(lst, norm)
    assert abs(float(norm) - want) <= 1.01 * ref.U * want
    mgn.mgn_grad_clip(lst, want / 7, norm.zero_())
    assert abs(float(norm) - want) <= 1.01 * ref.U * want
    h = ref.half(dtype)
    for a, b in zip(flat.split(1 << 25), out.split(1 << 25)):
        w = a.double() * (float(np.float32(want / 7)) / want)
        assert bool(((b.double() - w).abs() <= (4 * ref.U + 1.01 * h) * w.abs()).all())
