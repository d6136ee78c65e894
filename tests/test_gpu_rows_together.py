"""The row and time operators as they are used together, and where the
framework's own paths call them: the lockstep exchange in 8 bits, a rollout
with a gated memory and an 8-bit history, and a training window read from an
8-bit history (norm -> 8-bit rows -> recurrence and back)."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import row_ref as ref
import synth
from parity import local_inputs, say
from paper_2307_13592_amd.lockstep import Lockstep
from paper_2307_13592_amd.runner import GatedMemory, LatentCache, RmsNorm, Session
from synth import meshes

pytestmark = pytest.mark.gpu


def _lockstep(prec, l, K, **kw):
    mesh = meshes.sector(6, 16, 10, 4, seed=7)
    whole = local_inputs(mesh, 0, l, K, 2, 11, part=np.zeros(mesh.n_nodes, np.int32))
    part = mgn.mgn_partition_slabs(mesh.key, 4)
    graphs = [mgn.mgn_graph_build(mesh.send, mesh.recv, part, mesh.n_nodes, p) for p in range(4)]
    ef = synth.edge_features(mesh)
    own = [g["l2g"][:g["n_owned"]] for g in graphs]
    ls = Lockstep(l, K, 2, prec, part, graphs, [whole["nf"][o] for o in own], [ef[g["eperm"]] for g in graphs],
                  whole["params"], **kw)
    return ls, [whole["d_out"][o] for o in own]


def _through8(x):
    """Rows as an 8-bit exchange delivers them."""
    c = LatentCache(x.shape[0], x.shape[1])
    c.store(x.contiguous())
    return c.load(torch.empty_like(x, memory_format=torch.contiguous_format))


@pytest.mark.parametrize("prec,l", [("fp32", 64), ("bf16", 128), ("bf16", 256)])
def test_lockstep_exchange_in_8_bits(prec, l):
    say(f"[rows8] lockstep, 4 parts, l={l} {prec}")
    K = 3
    a, _ = _lockstep(prec, l, K)
    b, d_outs = _lockstep(prec, l, K, halo8=True)
    try:
        outs_a = [o.clone() for o in a.forward()]
        outs_b = [o.clone() for o in b.forward()]
        for sa, sb in zip(a.sessions, b.sessions):
            # the first block's halo comes from the encoders, which both share
            assert torch.equal(sb.halo[0], _through8(sa.halo[0]))
            # and every part's step is the step on the halo it received
            again = sb.forward()
            assert torch.equal(again, outs_b[b.sessions.index(sb)])
        num = sum(float((x - y).double().square().sum()) for x, y in zip(outs_a, outs_b))
        den = sum(float(x.double().square().sum()) for x in outs_a)
        e = (num / den) ** 0.5
        say(f"  outputs: {e:.2e} from the fp32 exchange")
        # an e4m3 row is off by at most 2^-4 of each value
        assert 0 < e <= ref.U8
    finally:
        a.close()
        b.close()


@pytest.mark.parametrize("prec,l", [("fp32", 64), ("bf16", 128)])
def test_lockstep_gradients_in_8_bits(prec, l):
    """One block: the owners take what the holders' gradients are worth in 8
    bits, link after link, and everything else stays as it was."""
    say(f"[rows8] lockstep gradients, l={l} {prec}")
    a, d_outs = _lockstep(prec, l, 1, halo8=True)
    b, _ = _lockstep(prec, l, 1, halo8=True, grads8=True)
    try:
        ds = [torch.as_tensor(np.ascontiguousarray(d)).cuda() for d in d_outs]
        a.forward()
        b.forward()
        got = b.backward(ds).clone()
        a.backward(ds)
        # the staged calls of a, with its halo gradients through 8 bits
        a.forward()
        for p, s in enumerate(a.sessions):
            mgn.mgn_backward_begin(s.model, ds[p], a.d_params, p > 0, s.d_halo)
        for s in a.sessions:
            mgn.mgn_backward_block(s.model)
        for p, q, recv, send in a.links:
            rows = _through8(a.sessions[p].d_halo[0][recv.long()])
            idx = torch.arange(rows.shape[0], dtype=torch.int32, device="cuda")
            mgn.mgn_add_latent_grads(a.sessions[q].model, rows, idx, send)
        for s in a.sessions:
            mgn.mgn_backward_end(s.model)
        assert torch.equal(got, a.d_params)
        for sa, sb in zip(a.sessions, b.sessions):
            assert torch.equal(sa.d_halo, sb.d_halo)
    finally:
        a.close()
        b.close()


def test_packed_latents_without_a_step():
    m = mgn.mgn_create(64, 1, 2)
    try:
        c = LatentCache(4, 64)
        rows = torch.arange(4, dtype=torch.int32, device="cuda")
        with pytest.raises(mgn.MgnError) as e:
            mgn.mgn_pack_latents8(m, rows, c.q, c.scale)
        assert e.value.status == mgn.MGN_E_STATE
        with pytest.raises(mgn.MgnError) as e:
            mgn.mgn_add_latent_grads8(m, c.q, c.scale, rows)
        assert e.value.status == mgn.MGN_E_STATE
        wide = LatentCache(4, 128)
        with pytest.raises(mgn.MgnError) as e:  # slots of another width than the latents
            mgn.mgn_pack_latents8(m, rows, wide.q, wide.scale)
        assert e.value.status == mgn.MGN_E_ARG
    finally:
        mgn.mgn_destroy(m)


def _session():
    mesh = meshes.delaunay_box(8, 7, 6, seed=3)
    c = local_inputs(mesh, 0, 64, 2, 2, 6, part=np.zeros(mesh.n_nodes, np.int32))
    return Session(64, 2, 2, "fp32", c["g"], c["nf"], c["ef"], c["halo"], c["params"], inference=True)


def test_rollout_with_memory_and_history():
    """A gate of -inf feeds the plain increments back (the rollout without a
    memory, bit for bit); a gate of 0 their half-half average; the history
    holds the outputs in 8 bits."""
    steps = 4
    s = _session()
    nf0 = s.node_feat.clone()
    try:
        n, d = s.out.shape
        outs = s.rollout(steps)
        end = s.node_feat.clone()
        s.node_feat.copy_(nf0)
        plain = s.rollout(steps, memory=GatedMemory(n, d, gate=torch.full((n, d), -float("inf"), device="cuda")))
        assert all(torch.equal(a, b) for a, b in zip(outs, plain)) and torch.equal(s.node_feat, end)
        s.node_feat.copy_(nf0)
        hist = LatentCache(steps * n, d)
        assert s.rollout(steps, history=hist) is hist
        assert torch.equal(s.node_feat, end)
        assert torch.equal(hist.load(torch.empty(steps * n, d, device="cuda")), _through8(torch.cat(outs)))
        s.node_feat.copy_(nf0)
        mem = GatedMemory(n, d, gate=torch.zeros(n, d, device="cuda"))
        outs = s.rollout(steps, memory=mem)
        h, q = torch.zeros(n, d, dtype=torch.float64, device="cuda"), nf0.double()[:, 3:3 + d]
        for o in outs:
            h = 0.5 * h + 0.5 * o.double()
            q = q + h
        assert torch.allclose(mem.state.double(), h, rtol=1e-6, atol=1e-6)
        assert torch.allclose(s.node_feat[:, 3:3 + d].double(), q, rtol=1e-5, atol=1e-5)
        with pytest.raises(ValueError):
            s.rollout(steps, history=LatentCache(n, d))
    finally:
        s.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_window_from_an_8_bit_history(dtype):
    """Each step's node rows (latents with a residual) are normalised into the
    history; the recurrence reads the window there; its gradient goes back
    through the norm.  Against the same chain in float64, each operator from
    the values that the one before it stored."""
    T, n, cols = 9, 300, 128
    say(f"[rows] history window {T} x {n} x {cols} {dtype}")
    r = torch.Generator(device="cuda")
    r.manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=r, device="cuda")
    v, res, g = rand(T, n, cols).to(dtype), rand(T, n, cols).to(dtype), rand(T, n, cols).to(dtype)
    norm, cache, mem = RmsNorm(cols), LatentCache(T * n, cols), GatedMemory(n, cols)
    norm.weight.copy_(1 + 0.1 * rand(cols))
    totals = [norm.store(v[t], cache, first=t * n, res=res[t]) for t in range(T)]
    q, scale = cache.window(0, T, n)
    h = mem.scan(g, q, x_scale=scale)
    x64 = ref.values8(q, scale)
    h64, e = ref.scan(ref.f64(g), x64, None, None)
    assert np.all(np.abs(ref.f64(h) - h64) <= e)
    # the same window step by step, as a rollout carries it
    m2 = GatedMemory(n, cols)
    for t in range(T):
        m2.step(q[t], g[t], scale[t])
    assert np.all(np.abs(ref.f64(m2.state) - h64[-1]) <= e[-1])
    dh = rand(T, n, cols)
    dg, dx, dh0 = mem.grad(g, q, h, dh, x_scale=scale)
    a, b, _, ea, eb, _ = ref.scan_grad(ref.f64(g), x64, ref.f64(h), ref.f64(mem.h0), None, ref.f64(dh), None)
    u = ref.half(dtype) + ref.U32
    assert np.all(np.abs(ref.f64(dg) - a) <= ea + np.abs(a) * u)
    assert np.all(np.abs(ref.f64(dx) - b) <= eb + np.abs(b) * u)
    dw = np.zeros(cols)
    mag = np.zeros(cols)
    for t in range(T):
        dt = norm.grad(totals[t], dx[t], accumulate=t > 0)
        want, w, slack, m = ref.rms_norm_grad(ref.f64(totals[t]), ref.f64(norm.weight), ref.f64(dx[t]), None, norm.eps)
        assert np.all(np.abs(ref.f64(dt) - want) <= slack + np.abs(want) * u)
        dw += w
        mag += m
    assert np.all(np.abs(ref.f64(norm.d_weight) - dw) <= mag * 64 * ref.U32 + np.abs(dw) * T * ref.U32)


def test_captured_step_carries_its_state():
    """A rollout's memory step recorded into a HIP graph: every replay moves
    the state on, as eager steps do."""
    n, cols = 500, 5
    gate = torch.randn(n, cols, device="cuda")
    x = torch.randn(n, cols, device="cuda")
    a, b = GatedMemory(n, cols, gate=gate), GatedMemory(n, cols, gate=gate)
    a.step(x)
    b.step(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.step(x)
    for k in range(4):
        x.copy_(torch.randn(n, cols, device="cuda"))
        g.replay()
        b.step(x)
        torch.cuda.synchronize()
        assert torch.equal(a.state, b.state), k


def test_calls_from_two_threads():
    """Two host threads, a stream each, calling at once (a long scan with
    scratch, and the norm's backward with its partials): everyone's own bits."""
    import threading
    T, rows, cols = 4000, 1, 64
    r = torch.Generator(device="cuda")
    r.manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=r, device="cuda")
    sets = [dict(g=rand(T, rows, cols), x=rand(T, rows, cols), t=rand(3000, 128), dy=rand(3000, 128)) for _ in range(2)]

    def run(s, stream):
        h = torch.empty(T, rows, cols, device="cuda")
        mgn.mgn_gated_scan(s["g"], s["x"], h=h, stream=stream)
        dx, dw = torch.empty_like(s["t"]), torch.empty(128, device="cuda")
        mgn.mgn_rms_norm_grad(s["t"], None, s["dy"], dx, dw, stream=stream)
        return h, dx, dw

    want = [run(s, None) for s in sets]
    torch.cuda.synchronize()
    got, bad = [None, None], []

    def work(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(20):
                    got[k] = run(sets[k], st.cuda_stream)
                    st.synchronize()
                    if not all(torch.equal(p, q) for p, q in zip(got[k], want[k])):
                        bad.append(k)
        except Exception as e:
            bad.append(e)

    ts = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    assert not bad, bad


def test_bindings_refuse_mismatched_tensors():
    x = torch.zeros(4, 128, device="cuda")
    w = torch.ones(128, device="cuda")
    q, s = torch.zeros(4, 128, dtype=torch.uint8, device="cuda"), torch.ones(4, 1, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    g = torch.zeros(3, 4, 128, device="cuda")
    for call in (lambda: mgn.mgn_rms_norm(x, w, x.cpu()), lambda: mgn.mgn_rms_norm(x, w[:64], x),
                 lambda: mgn.mgn_rms_norm(x, w, x, res=x.bfloat16()), lambda: mgn.mgn_rms_norm(x.t(), None, x.t()),
                 lambda: mgn.mgn_rms_norm_grad(x, w, x, None), lambda: mgn.mgn_rms_norm_grad(x, w, x[:3], x),
                 lambda: mgn.mgn_rows_store8(x, q, s, src_rows=i.long()),
                 lambda: mgn.mgn_rows_store8(x, q, s, src_rows=i, slots=i[:3]),
                 lambda: mgn.mgn_rows_store8(x, q, torch.ones(4, 2, device="cuda")),
                 lambda: mgn.mgn_rows_load8(q, s, x[:, :64].contiguous()),
                 lambda: mgn.mgn_gated_scan(g, g, h_last=x.bfloat16()), lambda: mgn.mgn_gated_scan(g, g[:2], h=g),
                 lambda: mgn.mgn_gated_scan(g, g, h=torch.empty_like(g), starts=torch.zeros(4, dtype=torch.uint8, device="cuda")),
                 lambda: LatentCache(4, 128).store(x, first=1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: mgn.mgn_rms_norm(x, w, q), lambda: mgn.mgn_rms_norm(x, w, x, y_scale=s),
                 lambda: mgn.mgn_rows_store8(x, q[:3], s[:3]), lambda: mgn.mgn_gated_scan(g, g),
                 lambda: mgn.mgn_rows_load8(q, s, x.bfloat16(), add=True)):
        with pytest.raises(mgn.MgnError) as e:
            call()
        assert e.value.status == mgn.MGN_E_ARG
