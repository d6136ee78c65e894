"""Rows in 8 bits (mgn_rows_store8, mgn_rows_load8) against the definition in
float64: the codes' values and the scales are equal, not near, since the scale
is a power of two and each value is rounded once."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref
from paper_2307_13592_amd.runner import LatentCache

pytestmark = pytest.mark.gpu


def _x(seed, n, cols, dtype=torch.float32):
    r = np.random.default_rng([seed, n, cols])
    x = r.standard_normal((n, cols)) * np.exp(3 * r.standard_normal((n, 1)))
    return torch.as_tensor(x.astype(np.float32)).to(dtype).cuda()


def _slots(n, cols):
    return (torch.full((n, cols), 0x55, dtype=torch.uint8, device="cuda"),
            torch.full((n, ref.blocks(cols)), 3.0, device="cuda"))


def _same(q, scale, x):
    want, ws = ref.store8(ref.f64(x))
    got = ref.values8(q, scale)
    assert np.array_equal(scale.cpu().numpy(), ws)
    assert np.array_equal(got, want, equal_nan=True), float(np.nanmax(np.abs(got - want)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", [(1, 1), (3, 5), (2, 7), (1, 16), (3, 6), (900, 5), (333, 11), (64, 8), (40, 16), (9, 9), (7, 64), (501, 17), (77, 21), (64, 32), (33, 48), (1885, 77), (33, 127), (130, 128), (65, 129), (9, 200),
                                    (1000, 256), (5, 257), (6, 1000), (3, 1024), (4, 1025), (2, 8192), (2, 8191)])
def test_store_and_load(n, cols, dtype):
    print(f"[rows8] {n} x {cols} {dtype}", flush=True)
    x = _x(1, n, cols, dtype)
    q, s = _slots(n, cols)
    mgn.mgn_rows_store8(x, q, s)
    _same(q, s, x)
    for out in (torch.float32, torch.bfloat16):
        y = torch.empty(n, cols, dtype=out, device="cuda")
        mgn.mgn_rows_load8(q, s, y)
        want = torch.as_tensor(ref.values8(q, s)).to(out)
        assert torch.equal(y.cpu(), want)
    # what was read back and stored again stands for the same values
    y = torch.empty(n, cols, device="cuda")
    mgn.mgn_rows_load8(q, s, y)
    q2, s2 = _slots(n, cols)
    mgn.mgn_rows_store8(y, q2, s2)
    y2 = torch.empty_like(y)
    mgn.mgn_rows_load8(q2, s2, y2)
    assert torch.equal(y, y2)


def test_every_code_reads_back():
    q = torch.arange(256, dtype=torch.uint8).view(2, 128).cuda()
    for scale in (1.0, 0.75, 2.0 ** -126, 2.0 ** 119):
        s = torch.full((2, 1), scale, device="cuda")
        y = torch.empty(2, 128, device="cuda")
        mgn.mgn_rows_load8(q, s, y)
        want = q.cpu().view(torch.float8_e4m3fn).float() * torch.tensor(scale)
        assert torch.equal(y.cpu().nan_to_num(nan=7e37), want.nan_to_num(nan=7e37)), scale
        z = torch.empty(2, 128, dtype=torch.bfloat16, device="cuda")
        mgn.mgn_rows_load8(q, s, z)
        assert torch.equal(z.cpu().float().nan_to_num(nan=7e37), want.bfloat16().float().nan_to_num(nan=7e37)), scale


@pytest.mark.parametrize("cols", [128, 130, 640])
def test_values_where_it_can_go_wrong(cols):
    """Blocks of zeros, infinities, NaNs, subnormal and huge magnitudes, and
    largest magnitudes at and beside 448 times a power of two."""
    print(f"[rows8] special values, {cols} columns", flush=True)
    rows = []
    r = np.random.default_rng(cols)

    def row(v):
        x = r.standard_normal(cols).astype(np.float32)
        x[:len(v)] = v
        rows.append(x)

    big = np.float32(3.4028235e38)
    rows.append(np.zeros(cols, np.float32))
    rows.append(np.full(cols, np.inf, np.float32))
    rows.append(np.full(cols, np.nan, np.float32))
    row([np.inf, -np.inf, np.nan, 1.0])
    row([big, -big, 1e-38])
    row([1e-45, -1e-45])
    rows.append(np.full(cols, 1e-42, np.float32))
    rows.append((r.standard_normal(cols) * 1e-38).astype(np.float32))
    for e in (-130, -118, -100, -1, 0, 1, 100, 119):
        for m in (1.75, np.nextafter(np.float32(1.75), np.float32(2)), np.nextafter(np.float32(1.75), np.float32(1)),
                  1.0, np.nextafter(np.float32(2), np.float32(1))):
            x = (r.uniform(-1, 1, cols) * m * 2.0 ** e).astype(np.float32)
            x[cols // 2] = np.float32(m * 2.0 ** e)
            rows.append(x)
    # halfway between codes: ties go to the even one
    ties = np.zeros(cols, np.float32)
    ties[:12] = [448, 17, 19, 21, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10, 0.015625, -17, -19]
    rows.append(ties)
    x = torch.as_tensor(np.stack(rows)).cuda()
    q, s = _slots(*x.shape)
    mgn.mgn_rows_store8(x, q, s)
    _same(q, s, x)


@pytest.mark.parametrize("cols", [5, 64, 77, 128, 256, 1030])
def test_index_lists(cols):
    """Gathered and scattered rows; pairs out of range are skipped and slots
    and rows that no pair names keep what they held."""
    print(f"[rows8] index lists, {cols} columns", flush=True)
    n_src, n_slots, n = 500, 700, 300
    r = np.random.default_rng(cols)
    x = _x(2, n_src, cols)
    src = r.integers(0, n_src, n).astype(np.int32)
    slots = r.permutation(n_slots)[:n].astype(np.int32)
    src[[0, 7, 8]] = [-1, n_src, 2 ** 31 - 1]
    slots[[20, 21, 22]] = [-5, n_slots, -2 ** 31]
    ok = (src >= 0) & (src < n_src) & (slots >= 0) & (slots < n_slots)
    dev = lambda a: torch.as_tensor(a).cuda()
    c = LatentCache(n_slots, cols)
    c.q.fill_(0x55)
    c.scale.fill_(3.0)
    c.store(x, src_rows=dev(src), slots=dev(slots))
    want, ws = ref.store8(ref.f64(x)[src[ok]])
    got = ref.values8(c.q, c.scale)
    assert np.array_equal(got[slots[ok]], want) and np.array_equal(c.scale.cpu().numpy()[slots[ok]], ws)
    rest = np.setdiff1d(np.arange(n_slots), slots[ok])
    assert bool((c.q.cpu()[rest] == 0x55).all()) and bool((c.scale.cpu()[rest] == 3.0).all())
    n_dst = 400
    rows = r.permutation(n_dst)[:n].astype(np.int32)
    rows[[30, 31]] = [-1, n_dst]
    ok2 = (slots >= 0) & (slots < n_slots) & (rows >= 0) & (rows < n_dst)
    for add in (False, True):
        base = torch.randn(n_dst, cols, device="cuda")
        dst = base.clone()
        c.load(dst, slots=dev(slots), dst_rows=dev(rows), add=add)
        w = base.cpu().numpy().copy()
        v = got[slots[ok2]].astype(np.float32)
        w[rows[ok2]] = w[rows[ok2]] + v if add else v
        assert np.array_equal(dst.cpu().numpy(), w), add
    # one list only: consecutive slots, or consecutive rows
    c.store(x, first=17, src_rows=dev(src[ok]))
    y = torch.zeros(int(ok.sum()), cols, device="cuda")
    c.load(y, first=17)
    assert np.array_equal(y.cpu().numpy().astype(np.float64), want)
    z = torch.zeros(n_dst, cols, device="cuda")
    c.load(z, first=17, dst_rows=torch.arange(int(ok.sum()) - 1, -1, -1, dtype=torch.int32, device="cuda"))
    assert torch.equal(z[:len(y)], y.flip(0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,cols", [(7, 128), (11, 64), (5, 260)])
def test_arrays_aligned_to_their_type_only(n, cols, dtype):
    print(f"[rows8] unaligned {n} x {cols} {dtype}", flush=True)
    x = _x(3, n, cols, dtype)
    q0, s0 = _slots(n, cols)
    mgn.mgn_rows_store8(x, q0, s0)
    y0 = torch.empty_like(x)
    mgn.mgn_rows_load8(q0, s0, y0)
    for ox, oq in ((1, 0), (0, 1), (3, 3), (0, 2)):
        xo = torch.empty(n * cols + 8, dtype=dtype, device="cuda")[ox:ox + n * cols].view(n, cols).copy_(x)
        buf = torch.full((n * cols + 8,), 0x55, dtype=torch.uint8, device="cuda")
        q = buf[oq:oq + n * cols].view(n, cols)
        s = torch.empty_like(s0)
        mgn.mgn_rows_store8(xo, q, s)
        assert torch.equal(q, q0) and torch.equal(s, s0)
        assert bool((buf[:oq] == 0x55).all()) and bool((buf[oq + n * cols:] == 0x55).all())
        wide = torch.full((n * cols + 8,), 9.0, dtype=dtype, device="cuda")
        y = wide[ox:ox + n * cols].view(n, cols)
        mgn.mgn_rows_load8(q, s, y)
        assert torch.equal(y, y0)
        assert bool((wide[:ox] == 9).all()) and bool((wide[ox + n * cols:] == 9).all())


@pytest.mark.parametrize("n,cols,dtype", [(1_000_003, 128, torch.float32), (1_500_001, 256, torch.bfloat16),
                                          (1_000_003, 77, torch.float32)])
def test_more_than_the_caches_hold(n, cols, dtype):
    print(f"[rows8] {n} x {cols} {dtype}", flush=True)
    x = (torch.randn(n, cols, device="cuda") * torch.exp(torch.randn(n, 1, device="cuda"))).to(dtype)
    q, s = _slots(n, cols)
    mgn.mgn_rows_store8(x, q, s)
    y = torch.empty_like(x)
    mgn.mgn_rows_load8(q, s, y)
    for b in range(ref.blocks(cols)):
        blk = x[:, b * 128:(b + 1) * 128].double()
        # (on the host: powers of two are exact there)
        m, e = np.frexp(blk.abs().amax(1, keepdim=True).cpu().numpy())
        p = torch.as_tensor(np.ldexp(1.0, e - 9 + (m > 0.875))).cuda()
        assert torch.equal(s[:, b:b + 1].double(), p)
        v = (blk / p).float().to(torch.float8_e4m3fn).double() * p
        assert torch.equal(y[:, b * 128:(b + 1) * 128].double(), v)


def test_offsets_past_32_bits():
    """Slots and rows whose offsets pass 2^31 and 2^32 elements."""
    cols, n_slots = 256, (1 << 24) + 5
    print("[rows8] 2^32 codes", flush=True)
    q = torch.zeros(n_slots, cols, dtype=torch.uint8, device="cuda")
    s = torch.ones(n_slots, 2, device="cuda")
    x = _x(5, 6, cols)
    at = torch.tensor([0, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24, n_slots - 1], dtype=torch.int32, device="cuda")
    mgn.mgn_rows_store8(x, q, s, slots=at)
    assert int((s != 1).any(1).sum()) <= 6 and int(q.any(1).sum()) == 6
    _same(q[at.long()], s[at.long()], x)
    y = torch.empty_like(x)
    mgn.mgn_rows_load8(q, s, y, slots=at)
    assert np.array_equal(ref.f64(y), ref.store8(ref.f64(x))[0])
    del q, s
    big = torch.zeros(n_slots, cols, dtype=torch.bfloat16, device="cuda")
    big[at.long()] = x.bfloat16()
    q, s = _slots(6, cols)
    mgn.mgn_rows_store8(big, q, s, src_rows=at)
    _same(q, s, x.bfloat16())
    mgn.mgn_rows_load8(q, s, big, dst_rows=at.flip(0))
    assert np.array_equal(ref.f64(big[at.long()]), ref.f64(torch.as_tensor(ref.values8(q, s)).flip(0).bfloat16()))


def test_no_rows():
    q, s = _slots(4, 128)
    mgn.mgn_rows_store8(torch.empty(0, 128, device="cuda"), q, s)
    mgn.mgn_rows_load8(q[:0], s[:0], torch.empty(3, 128, device="cuda"))
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    mgn.mgn_rows_store8(torch.empty(5, 128, device="cuda"), q, s, src_rows=e, slots=e)
    assert bool((q == 0x55).all()) and bool((s == 3.0).all())


def test_streams_and_captured_replays():
    """On a stream of its own, and replayed from a HIP graph with new inputs
    and eager work between the replays."""
    x = _x(7, 1000, 128)
    q, s = _slots(1000, 128)
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mgn.mgn_rows_store8(x, q, s, stream=side.cuda_stream)
    mgn.mgn_rows_load8(q, s, y, stream=side.cuda_stream)
    side.synchronize()
    _same(q, s, x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mgn.mgn_rows_store8(x, q, s)
        mgn.mgn_rows_load8(q, s, y)
    for k in range(4):
        x.copy_(_x(8 + k, 1000, 128))
        q.zero_()
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        _same(q, s, x)
        assert np.array_equal(ref.f64(y), ref.values8(q, s))
