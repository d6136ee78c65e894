"""The norm in its largest forms: a residual, its sum and every kind of row
written, past what the caches hold and past one turn of the grid, and its
backward with the residual's gradient.  Against float64 on the device; the bounds
are those of the small tests: 32 half-steps for y, 90 for the sums of dx."""
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref

pytestmark = pytest.mark.gpu
EPS = 1e-6
LARGE = [(1_200_001, 128), (600_001, 256), (1_000_003, 77), (60_001, 1100), (40_001, 4100), (40_001, 4099)]


def _rand(seed):
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    return lambda *s: torch.randn(s, generator=r, device="cuda")


def _parts(n, cols):
    """Row ranges whose float64 copies stay near 1 GB."""
    step = max(1, (1 << 27) // cols)
    return [slice(k, min(k + step, n)) for k in range(0, n, step)]


def _steps8(y64, cols):
    """The scale of every value's block of 128 columns."""
    out = torch.empty_like(y64)
    for b in range(0, cols, 128):
        a = y64[:, b:b + 128].abs().amax(1, keepdim=True)
        m, e = torch.frexp(a.float())  # (a power of two: one scale up or down is allowed for)
        out[:, b:b + 128] = torch.ldexp(torch.ones_like(a), e - 9 + (m > 0.875).int())
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", ["fp32", "bf16", "e4m3"])
@pytest.mark.parametrize("n,cols", LARGE)
def test_forward_with_residual(n, cols, out, dtype):
    print(f"[rms] {n} x {cols} {dtype} into {out}", flush=True)
    rand = _rand(n)
    x, res, w = rand(n, cols).to(dtype), rand(n, cols).to(dtype), 1 + 0.1 * rand(cols)
    x[n // 2] = res[n // 2] = 0
    total = torch.empty_like(x)
    scale = None
    if out == "e4m3":
        y = torch.full((n + 1, cols), 0x55, dtype=torch.uint8, device="cuda")
        scale = torch.full((n + 1, ref.blocks(cols)), 3.0, device="cuda")
        mgn.mgn_rms_norm(x, w, y[:n], res=res, total=total, y_scale=scale[:n], eps=EPS)
        assert bool((y[n] == 0x55).all()) and bool((scale[n] == 3).all())
        values = torch.empty(n, cols, device="cuda")
        mgn.mgn_rows_load8(y[:n], scale[:n], values)
        u = ref.U8
    else:
        values = torch.empty(n, cols, dtype=torch.float32 if out == "fp32" else torch.bfloat16, device="cuda")
        mgn.mgn_rms_norm(x, w, values, res=res, total=total, eps=EPS)
        u = ref.half(values.dtype)
    for p in _parts(n, cols):
        t = x[p].double() + res[p].double()
        # t: rounded to fp32, then to its type
        assert bool(((total[p].double() - t).abs() <= t.abs() * (ref.U32 + (ref.U16 if dtype == torch.bfloat16 else 0)) *
                     (1 + 2.0 ** -7)).all())
        y64 = t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * w.double()
        bound = y64.abs() * (u + 34 * ref.U32) + 1e-37
        if out == "e4m3":
            bound += 2 * _steps8(y64, cols) * 2.0 ** -10
        assert bool(((values[p].double() - y64).abs() <= bound).all())
        del t, y64, bound


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", LARGE)
def test_backward_with_d_total(n, cols, dtype):
    print(f"[rms grad] {n} x {cols} {dtype}", flush=True)
    rand = _rand(n + 1)
    t, dy, ds, w = rand(n, cols).to(dtype), rand(n, cols).to(dtype), rand(n, cols).to(dtype), 1 + 0.1 * rand(cols)
    dx, dw = torch.empty_like(t), torch.empty(cols, device="cuda")
    mgn.mgn_rms_norm_grad(t, w, dy, dx, dw, d_total=ds, eps=EPS)
    sums = torch.zeros(2, cols, dtype=torch.float64, device="cuda")
    for p in _parts(n, cols):
        v, g = t[p].double(), dy[p].double()
        inv = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
        u, wg = v * inv, g * w.double()
        want = (wg - u * (u * wg).mean(1, keepdim=True)) * inv + ds[p].double()
        slack = (wg.abs() + u.abs() * (u * wg).abs().mean(1, keepdim=True)) * inv * 90 * ref.U32
        slack += want.abs() * (ref.half(dtype) + 4 * ref.U32)
        assert bool(((dx[p].double() - want).abs() <= slack).all())
        sums += torch.stack([(g * u).sum(0), (g * u).abs().sum(0)])
        del v, g, u, wg, want, slack
    # u within 32 half-steps, a product, 8 rows in fp32, a partial, the result
    assert bool(((dw.double() - sums[0]).abs() <= sums[1] * (32 + 1 + 8 + 1) * ref.U32 + sums[0].abs() * ref.U32).all())
