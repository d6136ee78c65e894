"""Refusals of the layer norm, the operators along time and gradient clipping: bad
sizes, types, pointers, overlaps and scratch are reported before anything is launched
(no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2307_13592_amd as mgn

P = [C.c_void_p((k + 1) << 34) for k in range(32)]  # far apart, never read
ODD, HALF = C.c_void_p((40 << 34) + 1), C.c_void_p((40 << 34) + 2)
INF, NAN = float("inf"), float("nan")
F32, BF16, E4M3 = mgn.MGN_FP32, mgn.MGN_BF16, mgn.MGN_E4M3


def _refused(st, what=None, status=mgn.MGN_E_ARG):
    assert st == status, st
    if what:
        assert what in mgn.mgn_last_error(None), mgn.mgn_last_error(None)


def test_layer_norm_refusals():
    L = mgn.lib()
    norm = lambda x=P[0], res=P[1], t=F32, rows=9, cols=128, w=P[2], b=P[3], eps=1e-5, total=P[4], y=P[5], yt=F32, ys=None: \
        L.mgn_layer_norm(x, res, t, rows, cols, w, b, eps, total, y, yt, ys, None)
    for kw in (dict(cols=0), dict(cols=8193), dict(rows=-1), dict(rows=1 << 60)):
        _refused(norm(**kw), "sizes")
    for kw in (dict(t=E4M3), dict(t=9), dict(yt=5)):
        _refused(norm(**kw), "type")
    for eps in (0.0, -1e-5, NAN, INF, 1e-40):
        _refused(norm(eps=eps), "eps")
    _refused(norm(yt=E4M3), "y_scale")
    _refused(norm(ys=P[6]), "y_scale")
    for kw in (dict(x=None), dict(y=None)):
        _refused(norm(**kw), "NULL")
    for k in ("x", "res", "w", "b", "total", "y"):
        _refused(norm(**{k: HALF}), "misaligned")
    for kw in (dict(total=P[5]), dict(y=P[2]), dict(total=P[3]), dict(y=C.c_void_p(P[0].value + 4)), dict(y=P[0], yt=BF16),
               dict(total=C.c_void_p(P[1].value + 512)), dict(x=P[2], total=P[2]), dict(y=P[3])):
        _refused(norm(**kw), "overlapping")
    assert norm(rows=0, x=None, y=None) == mgn.MGN_OK

    grad = lambda total=P[0], t=F32, w=P[1], eps=1e-5, dy=P[2], ds=P[3], rows=9, cols=128, dx=P[4], dw=P[5], db=P[6], work=P[7]: \
        L.mgn_layer_norm_grad(total, t, w, eps, dy, ds, rows, cols, dx, dw, db, 0, work, None)
    for kw in (dict(cols=0), dict(rows=-1)):
        _refused(grad(**kw), "sizes")
    _refused(grad(t=E4M3), "type")
    _refused(grad(eps=0.0), "eps")
    for kw in (dict(total=None), dict(dy=None), dict(dx=None)):
        _refused(grad(**kw), "NULL")
    for kw in (dict(work=None), dict(work=None, dw=None)):
        _refused(grad(**kw), "work")
    for k in ("total", "w", "dy", "ds", "dx", "dw", "db", "work"):
        _refused(grad(**{k: HALF}), "misaligned")
    for kw in (dict(dx=C.c_void_p(P[0].value + 4)), dict(dw=P[6]), dict(dw=P[1]), dict(work=P[4]), dict(db=P[2]),
               dict(work=C.c_void_p(P[5].value - 4 * 2048 * 128 + 4)), dict(dx=P[1])):
        _refused(grad(**kw), "overlapping")


def test_causal_conv_refusals():
    L = mgn.lib()
    conv = lambda x=P[0], t=F32, w=P[1], W=4, b=P[2], st=P[3], past=P[4], T=7, rows=5, cols=64, y=P[5], out=P[6]: \
        L.mgn_causal_conv(x, t, w, W, b, st, past, T, rows, cols, 1, y, out, None)
    for W in (0, 9, -1):
        _refused(conv(W=W), "width")
    for kw in (dict(cols=0), dict(cols=8193), dict(rows=-1), dict(T=-1), dict(T=1 << 50)):
        _refused(conv(**kw), "sizes")
    _refused(conv(t=E4M3), "type")
    for kw in (dict(x=None), dict(w=None), dict(y=None)):
        _refused(conv(**kw), "NULL")
    for k in ("x", "w", "b", "past", "y", "out"):
        _refused(conv(**{k: HALF}), "misaligned")
    for kw in (dict(y=P[0]), dict(out=P[0]), dict(y=P[4]), dict(out=C.c_void_p(P[4].value + 4)), dict(out=P[5]), dict(y=P[3]),
               dict(out=P[1])):
        _refused(conv(**kw), "overlapping")
    assert conv(rows=0, x=None, y=None) == mgn.MGN_OK and conv(T=0, out=None) == mgn.MGN_OK
    assert conv(T=0, W=1) == mgn.MGN_OK  # one tap: nothing before it

    grad = lambda x=P[0], t=F32, w=P[1], W=4, b=P[2], st=P[3], past=P[4], dy=P[5], dpo=P[6], T=7, rows=5, cols=64, dx=P[7], \
        dw=P[8], db=P[9], dp=P[10], work=P[11]: \
        L.mgn_causal_conv_grad(x, t, w, W, b, st, past, dy, dpo, T, rows, cols, 1, dx, dw, db, 0, dp, work, None)
    _refused(grad(W=9), "width")
    _refused(grad(T=-1), "sizes")
    _refused(grad(t=7), "type")
    for kw in (dict(x=None), dict(w=None), dict(dy=None), dict(dx=None)):
        _refused(grad(**kw), "NULL")
    _refused(grad(work=None), "work")
    for k in ("x", "w", "b", "past", "dy", "dpo", "dx", "dw", "db", "dp", "work"):
        _refused(grad(**{k: HALF}), "misaligned")
    for kw in (dict(dx=P[5]), dict(dx=P[0]), dict(dp=P[6]), dict(dw=P[9]), dict(dw=P[1]), dict(work=P[4]), dict(db=P[2])):
        _refused(grad(**kw), "overlapping")


def _ssm(T=7, rows=5, cols=64, n=16, t=F32, x=P[0], dt=P[1], B=P[2], Cn=P[3], z=P[4], A=P[5], D=P[6], b=P[7], st=P[8]):
    return mgn.mgn_ssm(T, rows, cols, n, t, 1, x, dt, B, Cn, z, A, D, b, st)


def test_selective_scan_refusals():
    L = mgn.lib()

    def scan(h0=P[9], y=P[10], last=P[11], marks=P[12], work=P[13], wb=1 << 30, **kw):
        return L.mgn_selective_scan(C.byref(_ssm(**kw)), h0, y, last, marks, work, wb, None)

    def grad(marks=P[9], dy=P[10], dl=P[11], dh0=P[12], work=P[13], wb=1 << 30, dx=P[14], ddt=P[15], dB=P[16], dC=P[17], dz=P[18],
             dA=P[19], dD=P[20], db=P[21], **kw):
        g = mgn.mgn_ssm_grads(dx, ddt, dB, dC, dz, dA, dD, db, 0)
        return L.mgn_selective_scan_grad(C.byref(_ssm(**kw)), marks, dy, dl, C.byref(g), dh0, work, wb, None)

    for call in (scan, grad):
        for n in (0, 65, -1):
            _refused(call(n=n), "n must be")
        for kw in (dict(cols=0), dict(cols=8193), dict(rows=-1), dict(T=-1), dict(T=1 << 50), dict(rows=1 << 45)):
            _refused(call(**kw), "sizes")
        _refused(call(t=E4M3), "type")
        for k in ("x", "dt", "B", "Cn", "A"):
            _refused(call(**{k: None}), "NULL")
        for k in ("x", "dt", "B", "Cn", "z", "A", "D", "b", "marks", "work"):
            _refused(call(**{k: HALF}), "misaligned")
        _refused(call(work=C.c_void_p(P[13].value + 8)), "misaligned")
    _refused(L.mgn_selective_scan(None, None, P[0], None, None, None, 0, None), "NULL")
    _refused(L.mgn_selective_scan_grad(None, P[0], P[1], None, None, None, None, 0, None), "NULL")
    _refused(L.mgn_selective_scan_grad(C.byref(_ssm()), P[9], P[10], None, None, None, P[13], 1 << 30, None), "NULL")
    _refused(scan(y=None), "NULL")
    for k in ("y", "h0", "last"):
        _refused(scan(**{k: HALF}), "misaligned")
    for kw in (dict(y=P[0]), dict(y=P[4]), dict(last=C.c_void_p(P[9].value + 4)), dict(marks=P[9]), dict(marks=P[11]), dict(last=P[5]),
               dict(y=P[12]), dict(y=P[8])):
        _refused(scan(**kw), "overlapping")
    for kw in (dict(marks=None), dict(dy=None), dict(dx=None), dict(ddt=None), dict(dB=None), dict(dC=None)):
        _refused(grad(**kw), "NULL")
    _refused(grad(dz=None), "dz")
    _refused(grad(z=None), "dz")
    for k in ("dy", "dl", "dh0", "dx", "ddt", "dB", "dC", "dz", "dA", "dD", "db"):
        _refused(grad(**{k: HALF}), "misaligned")
    for kw in (dict(dx=P[10]), dict(dx=P[0]), dict(dB=P[17]), dict(dB=P[2]), dict(dh0=P[9]), dict(dA=P[5]), dict(dD=P[21]),
               dict(work=P[9]), dict(dh0=C.c_void_p(P[11].value + 64)), dict(ddt=P[1])):
        _refused(grad(**kw), "overlapping")
    # scratch
    b = C.c_size_t()
    for f, call in ((L.mgn_selective_scan_work, scan), (L.mgn_selective_scan_grad_work, grad)):
        assert f(5000, 1, 64, 16, C.byref(b)) == mgn.MGN_OK and b.value > 0
        _refused(call(T=5000, rows=1, wb=b.value - 1), "work", mgn.MGN_E_NOMEM)
        _refused(call(T=5000, rows=1, work=None, wb=b.value), "work", mgn.MGN_E_NOMEM)
        _refused(f(1, 1, 1, 1, None), "NULL")
        _refused(f(1, 1, 1, 65, C.byref(b)), "n must be")
        _refused(f(-1, 1, 1, 1, C.byref(b)), "sizes")
        assert f(0, 5, 64, 16, C.byref(b)) == mgn.MGN_OK and b.value == 0
    assert L.mgn_selective_scan_work(20, 100000, 64, 16, C.byref(b)) == mgn.MGN_OK and b.value == 0


def test_gradient_list_refusals():
    L = mgn.lib()

    def create(*tensors):
        rec = (mgn.mgn_grad * max(len(tensors), 1))(*[mgn.mgn_grad(*t) for t in tensors])
        p = C.c_void_p()
        st = L.mgn_grads_create(rec, len(tensors), C.byref(p))
        return st, p

    a, b, c = (p.value for p in P[:3])
    for t in ((a, None, 5, E4M3), (a, None, 5, 9)):
        _refused(create(t)[0], "type")
    for t in ((a, None, -1, F32), (a, None, 1 << 50, F32), (a, None, 1 << 40, F32)):
        _refused(create(t)[0], "sizes")
    _refused(create((None, b, 5, F32))[0], "NULL")
    _refused(create((a + 2, None, 5, F32))[0], "misaligned")
    _refused(create((a, b + 1, 5, BF16))[0], "misaligned")
    for t in ((1 << 48, None, 5, F32), (a, 1 << 60, 5, F32)):
        _refused(create(t)[0], "device address")
    for ts in ([(a, None, 5, F32), (a, None, 5, F32)], [(a, None, 5, F32), (a + 16, b, 5, F32)], [(a, a + 4, 5, F32)],
               [(a, b, 5, F32), (c, b + 8, 5, F32)], [(a, b, 5, F32), (b, c, 5, F32)], [(a, c, 50, F32), (a + 40, a + 400, 5, BF16), (b, a + 100, 3, F32)]):
        _refused(create(*ts)[0], "overlapping")
    _refused(L.mgn_grads_create(None, 1, C.byref(C.c_void_p())), "NULL")
    _refused(L.mgn_grads_create(None, 0, None), "NULL")
    st, p = create((a, b, 5, F32), (a, c, 5, F32), (None, None, 0, BF16))  # read twice
    assert st == mgn.MGN_OK
    n = C.c_size_t()
    assert L.mgn_grads_work(p, C.byref(n)) == mgn.MGN_OK and n.value > 0
    _refused(L.mgn_grads_work(None, C.byref(n)), "NULL")
    _refused(L.mgn_grad_norm(p, None, P[5], n.value, None), "NULL")
    _refused(L.mgn_grad_norm(None, P[4], P[5], n.value, None), "NULL")
    _refused(L.mgn_grad_norm(p, P[4], P[5], n.value - 1, None), "work", mgn.MGN_E_NOMEM)
    _refused(L.mgn_grad_norm(p, P[4], None, n.value, None), "work", mgn.MGN_E_NOMEM)
    _refused(L.mgn_grad_norm(p, HALF, P[5], n.value, None), "misaligned")
    _refused(L.mgn_grad_norm(p, P[0], P[5], n.value, None), "overlapping")
    _refused(L.mgn_grad_clip(p, 1.0, 0, P[4], P[1], n.value, None), "overlapping")
    _refused(L.mgn_grad_clip(p, 1.0, 0, P[5], P[5], n.value, None), "overlapping")
    for most in (0.0, -1.0, NAN, INF):
        _refused(L.mgn_grad_clip(p, most, 0, P[4], P[5], n.value, None), "max_norm")
    L.mgn_grads_destroy(p)
    L.mgn_grads_destroy(None)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, w = torch.zeros(3, 4), torch.ones(4)
    with pytest.raises(ValueError):
        mgn.mgn_layer_norm(x, w, w, x.clone())
    with pytest.raises(ValueError):
        mgn.mgn_layer_norm_grad(x, w, x, x.clone(), w.clone())
    s = torch.zeros(2, 3, 4)
    for bad in (torch.ones(4), torch.ones(4, 0), torch.ones(4, 9), torch.ones(5, 4)):
        with pytest.raises(ValueError):
            mgn.mgn_causal_conv(s, bad, s.clone())
    with pytest.raises(ValueError):
        mgn.mgn_causal_conv(s, torch.ones(4, 4), s.clone())
    for A in (torch.ones(4), torch.ones(4, 65), torch.ones(4, 0), None):
        with pytest.raises(ValueError):
            mgn.mgn_selective_scan(s, s, A, s, s, s.clone())
    with pytest.raises(ValueError):
        mgn.mgn_selective_scan(s, s, torch.ones(4, 2), torch.zeros(2, 3, 2), torch.zeros(2, 3, 2), s.clone())
    with pytest.raises(ValueError):
        mgn.mgn_grad_norm([torch.zeros(3)], torch.zeros(1))
    with pytest.raises(ValueError):
        mgn.mgn_grad_list([torch.zeros(3)])
    with pytest.raises(ValueError):
        mgn.mgn_grad_list([torch.zeros(3)], [None, None])
    with pytest.raises(ValueError):
        mgn.mgn_grad_list([torch.zeros(3, dtype=torch.float16)])
