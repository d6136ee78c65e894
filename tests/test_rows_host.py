"""Refusals of the row and time operators: bad sizes, types, pointers, overlaps
and scratch are reported before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2307_13592_amd as mgn

P = [C.c_void_p((k + 1) << 32) for k in range(16)]  # far apart, never read
ODD = C.c_void_p((40 << 32) + 1)
HALF = C.c_void_p((40 << 32) + 2)
INF, NAN = float("inf"), float("nan")
F32, BF16, E4M3 = mgn.MGN_FP32, mgn.MGN_BF16, mgn.MGN_E4M3


def _refused(st, what=None, status=mgn.MGN_E_ARG):
    assert st == status, st
    if what:
        assert what in mgn.mgn_last_error(None)


def test_rows8_refusals():
    L = mgn.lib()
    store = lambda src=P[0], t=F32, n_src=9, cols=128, rows=P[1], slots=P[2], n=5, q=P[3], s=P[4], n_slots=7: \
        L.mgn_rows_store8(src, t, n_src, cols, rows, slots, n, q, s, n_slots, None)
    load = lambda q=P[0], s=P[1], n_slots=9, cols=128, slots=P[2], rows=P[3], n=5, dst=P[4], t=F32, n_dst=7, add=0: \
        L.mgn_rows_load8(q, s, n_slots, cols, slots, rows, n, dst, t, n_dst, add, None)
    for call in (store, load):
        for kw in (dict(cols=0), dict(cols=8193), dict(cols=-1)):
            _refused(call(**kw), "cols")
        for kw in (dict(t=E4M3), dict(t=7), dict(t=-1)):
            _refused(call(**kw), "type")
        for kw in (dict(n=-1), dict(n_slots=-1), dict(n=1 << 60)):
            _refused(call(**kw), "sizes")
        for kw in (dict(q=None), dict(s=None)):
            _refused(call(**kw), "NULL")
        for kw in (dict(s=HALF), dict(rows=HALF), dict(slots=ODD)):
            _refused(call(**kw), "misaligned")
        assert call(n=0) == mgn.MGN_OK
    _refused(store(src=None), "NULL")
    _refused(load(dst=None), "NULL")
    _refused(store(src=HALF), "misaligned")
    _refused(store(src=ODD, t=BF16), "misaligned")
    _refused(load(dst=ODD, t=BF16), "misaligned")
    _refused(store(rows=None, n=10, n_slots=20), "more rows")
    _refused(store(slots=None, n=8), "more rows")
    _refused(load(rows=None, n=8), "more rows")
    _refused(load(slots=None, n=10, n_dst=20), "more rows")
    _refused(load(t=BF16, add=1), "MGN_FP32 only")
    _refused(store(q=C.c_void_p(P[0].value + 64)), "overlapping")
    _refused(store(s=C.c_void_p(P[3].value + 4)), "overlapping")
    _refused(load(dst=C.c_void_p(P[1].value - 4)), "overlapping")


def test_rms_norm_refusals():
    L = mgn.lib()
    fwd = lambda x=P[0], res=P[1], t=F32, rows=5, cols=128, w=P[2], eps=1e-6, tot=P[3], y=P[4], yt=F32, s=None: \
        L.mgn_rms_norm(x, res, t, rows, cols, w, eps, tot, y, yt, s, None)
    bwd = lambda tot=P[0], t=F32, w=P[1], eps=1e-6, dy=P[2], ds=P[3], rows=5, cols=128, dx=P[4], dw=P[5], acc=0, wk=P[6]: \
        L.mgn_rms_norm_grad(tot, t, w, eps, dy, ds, rows, cols, dx, dw, acc, wk, None)
    for call in (fwd, bwd):
        for kw in (dict(cols=0), dict(cols=8193), dict(rows=-1), dict(rows=1 << 50)):
            _refused(call(**kw), "sizes")
        for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(eps=1e-40)):
            _refused(call(**kw), "eps")
        _refused(call(t=E4M3), "type")
        _refused(call(w=HALF), "misaligned")
    for kw in (dict(x=None), dict(y=None)):
        _refused(fwd(**kw), "NULL")
    for kw in (dict(x=HALF), dict(res=HALF), dict(tot=ODD), dict(y=ODD, yt=BF16), dict(y=P[4], yt=E4M3, s=HALF)):
        _refused(fwd(**kw), "misaligned")
    _refused(fwd(yt=3), "type")
    _refused(fwd(yt=E4M3), "y_scale")
    _refused(fwd(s=P[5]), "y_scale")
    for kw in (dict(tot=P[4]), dict(y=P[0], tot=P[0]), dict(y=P[0], yt=BF16), dict(y=C.c_void_p(P[0].value + 4)),
               dict(tot=C.c_void_p(P[1].value + 512)), dict(y=P[2]), dict(x=C.c_void_p(P[1].value + 4), tot=P[1])):
        _refused(fwd(**kw), "overlapping")
    assert fwd(rows=0) == mgn.MGN_OK
    for kw in (dict(tot=None), dict(dy=None), dict(dx=None)):
        _refused(bwd(**kw), "NULL")
    _refused(bwd(wk=None), "needs work")
    for kw in (dict(dx=C.c_void_p(P[2].value + 4)), dict(dw=P[6]), dict(wk=P[0]), dict(dw=P[1]),
               dict(dx=P[2], ds=C.c_void_p(P[2].value + 16))):
        _refused(bwd(**kw), "overlapping")
    assert bwd(rows=0, dw=None) == mgn.MGN_OK


def test_gated_scan_refusals():
    L = mgn.lib()
    n = C.c_size_t()
    assert L.mgn_gated_scan_work(7, 5, 128, C.byref(n)) == mgn.MGN_OK
    _refused(L.mgn_gated_scan_work(7, 5, 128, None), "NULL")
    fwd = lambda g=P[0], gt=F32, x=P[1], xt=F32, xs=None, st=P[2], h0=P[3], T=7, rows=5, cols=128, h=P[4], last=P[5], \
        wk=P[6], nb=1 << 31: L.mgn_gated_scan(g, gt, x, xt, xs, st, h0, T, rows, cols, h, last, wk, nb, None)
    bwd = lambda g=P[0], gt=F32, x=P[1], xt=F32, xs=None, st=P[2], h0=P[3], h=P[4], dh=P[5], dl=P[6], T=7, rows=5, \
        cols=128, dg=P[7], dx=P[8], d0=P[9], wk=P[10], nb=1 << 31: \
        L.mgn_gated_scan_grad(g, gt, x, xt, xs, st, h0, h, dh, dl, T, rows, cols, dg, dx, d0, wk, nb, None)
    for call in (fwd, bwd):
        for kw in (dict(cols=0), dict(cols=8193), dict(rows=-1), dict(T=-1), dict(T=1 << 50)):
            _refused(call(**kw), "sizes")
        for kw in (dict(gt=E4M3), dict(gt=5), dict(xt=BF16), dict(xt=9), dict(gt=BF16)):
            _refused(call(**kw), "must be")
        for kw in (dict(xt=E4M3), dict(xs=P[11])):
            _refused(call(**kw), "x_scale")
        for kw in (dict(g=None), dict(x=None)):
            _refused(call(**kw), "NULL")
        for kw in (dict(g=HALF), dict(x=HALF), dict(h0=HALF), dict(xt=E4M3, xs=HALF), dict(wk=C.c_void_p(P[6].value + 8)),
                   dict(h=HALF)):
            _refused(call(**kw), "misaligned")
        assert call(rows=0) == mgn.MGN_OK
    _refused(fwd(h=None, last=None), "neither")
    _refused(fwd(last=HALF), "misaligned")
    for kw in (dict(h=P[0]), dict(last=P[1]), dict(h=C.c_void_p(P[3].value + 4)), dict(last=C.c_void_p(P[3].value + 4)),
               dict(h=P[5]), dict(last=C.c_void_p(P[4].value + 16)), dict(h=P[2])):
        _refused(fwd(**kw), "overlapping")
    assert fwd(T=0, last=None) == mgn.MGN_OK
    for kw in (dict(h=None), dict(dg=None), dict(dx=None)):
        _refused(bwd(**kw), "NULL")
    for kw in (dict(dg=P[0]), dict(dx=P[1]), dict(dg=P[8]), dict(d0=P[3]), dict(d0=C.c_void_p(P[6].value + 4)),
               dict(dx=P[5]), dict(dg=P[4])):
        _refused(bwd(**kw), "overlapping")
    assert bwd(T=0, d0=None) == mgn.MGN_OK
    # few columns over many steps need scratch
    need = mgn.mgn_gated_scan_work(100_000, 1, 64)
    if need:
        _refused(fwd(T=100_000, rows=1, cols=64, wk=None), "work", mgn.MGN_E_NOMEM)
        _refused(fwd(T=100_000, rows=1, cols=64, nb=need - 1), "work", mgn.MGN_E_NOMEM)
        _refused(bwd(T=100_000, rows=1, cols=64, nb=need - 1), "work", mgn.MGN_E_NOMEM)


def test_exchange_refusals():
    L = mgn.lib()
    h = mgn.mgn_create(64, 2, 2)
    h2 = mgn.mgn_create(64, 2, 2)
    try:
        assert L.mgn_pack_latents8(None, P[0], 3, P[1], P[2], 64, None) == mgn.MGN_E_ARG
        assert L.mgn_add_latent_grads8(None, P[1], P[2], 64, P[0], 3, None) == mgn.MGN_E_ARG
        assert L.mgn_pack_latents8(h, P[0], 3, P[1], P[2], 128, None) == mgn.MGN_E_ARG
        assert L.mgn_pack_latents8(h, P[0], -1, P[1], P[2], 64, None) == mgn.MGN_E_ARG
        assert L.mgn_pack_latents8(h, P[0], 3, None, P[2], 64, None) == mgn.MGN_E_ARG
        assert L.mgn_pack_latents8(h, P[0], 3, P[1], HALF, 64, None) == mgn.MGN_E_ARG
        assert L.mgn_pack_latents8(h, P[0], 3, P[1], P[2], 64, None) == mgn.MGN_E_STATE
        assert L.mgn_add_latent_grads8(h, P[1], P[2], 128, P[0], 3, None) == mgn.MGN_E_ARG
        assert L.mgn_add_latent_grads8(h, P[1], P[2], 64, P[0], 3, None) == mgn.MGN_E_STATE
        ms = (C.c_void_p * 2)(h.value, h2.value)
        ok = (mgn.mgn_halo_link * 1)(mgn.mgn_halo_link(0, 1, P[0], P[1], 3))
        d = (C.c_void_p * 2)(P[2].value, P[3].value)
        fwd = lambda q=P[4], s=P[5], slots=3, cols=64: L.mgn_lockstep_forward8(2, ms, None, d, d, d, d, d, None, ok, 1,
                                                                              q, s, slots, cols, None)
        bwd = lambda q=P[4], s=P[5], slots=3, cols=64: L.mgn_lockstep_backward8(2, ms, d, P[6], 0, d, ok, 1, q, s, slots,
                                                                               cols, None)
        for call in (fwd, bwd):
            _refused(call(slots=2), "more rows")
            _refused(call(slots=-1), "sizes")
            _refused(call(cols=128), "sizes")
            _refused(call(q=None), "scratch")
            _refused(call(s=HALF), "scratch")
        _refused(fwd(), "NULL array")
        assert bwd() == mgn.MGN_E_STATE
    finally:
        mgn.mgn_destroy(h)
        mgn.mgn_destroy(h2)


def test_bindings_refuse_what_the_abi_cannot_see():
    x = torch.zeros(4, 128)
    q, s = torch.zeros(4, 128, dtype=torch.uint8), torch.ones(4, 1)
    for call in (lambda: mgn.mgn_rows_store8(x, q, s),  # host tensors
                 lambda: mgn.mgn_rows_store8(x.double(), q, s),
                 lambda: mgn.mgn_rows_store8(x[0], q, s),
                 lambda: mgn.mgn_rows_load8(q, s, x),
                 lambda: mgn.mgn_rms_norm(x, None, x.half()),
                 lambda: mgn.mgn_rms_norm(x[0], None, x),
                 lambda: mgn.mgn_rms_norm_grad(x, None, x, x),
                 lambda: mgn.mgn_gated_scan(x, x),
                 lambda: mgn.mgn_gated_scan(x[None], x[None].bfloat16()),
                 lambda: mgn.mgn_gated_scan(x[None], x[None])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(mgn.MgnError):
        mgn.mgn_gated_scan_work(-1, 5, 64)
