"""What a trajectory's memory is made of and trained with, as it is measured:
the layer norm of node rows with the residual's addition, the short causal
convolution and the selective state space scan over time steps, each forward
and backward, and the global gradient norm with clipping over many tensors.

A case is a dict of plain values:
  op      "ln", "ln_grad", "conv", "conv_grad", "ssm" (forward: a whole
          trajectory, or one step of a rollout), "ssm_train" (forward and
          backward), "clip"
  rows    node rows; cols  columns of a row; steps  time steps
  type    storage type of the inputs, "fp32" or "bf16"; out  that of the
          norm's result
  res     the norm adds a residual (its gradient: one more gradient arrives
          at the sum)
  width   taps of the convolution; silu  it ends in x sigmoid(x)
  n       states a column
  gate    the scan's result is multiplied by z sigmoid(z)
  starts  share of time steps that begin a new trajectory
  state   what came before the steps is given, and what they leave is wanted
          (its gradient: one arrives at what they leave)
  sizes   clip: "model" (the tensors of the network with `layers` blocks and
          latent `cols`) or "even" (`layers` tensors of about `rows` values)
  over    clip: the norm is this many times the largest allowed one
"""
import math

import torch

own = False

EPS = 1e-5
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one layer's norm on a few boundary rows: the call's latency
        dict(name="ln_few", op="ln", rows=33, cols=64, type="fp32", out="fp32", res=True),
        # the 2M-node partition's bf16 latents with the residual stream
        dict(name="ln_mesh", op="ln", rows=2000000, cols=128, type="bf16", out="bf16", res=True),
        # the 1M-node fp32 partition in training: backward with the residual stream's gradient
        dict(name="ln_mesh_grad", op="ln_grad", rows=1000000, cols=128, type="fp32", res=True),
        # a 20-step window of a large mesh's bf16 latents, several short trajectories in it
        dict(name="conv_window", op="conv", steps=20, rows=100003, cols=64, type="bf16", width=4, silu=True, starts=0.15, state=False),
        # a 600-step cylinder trajectory, backward
        dict(name="conv_cylinder_grad", op="conv_grad", steps=600, rows=1885, cols=128, type="fp32", width=4, silu=True, starts=0.0, state=True),
        # one rollout step on the cylinder mesh (1,885 nodes): the state is carried
        dict(name="ssm_step", op="ssm", steps=1, rows=1885, cols=128, n=16, type="fp32", gate=True, starts=0.0, state=True),
        # a 600-step cylinder trajectory
        dict(name="ssm_cylinder", op="ssm", steps=600, rows=1885, cols=64, n=16, type="bf16", gate=True, starts=0.0, state=False),
        # three probes over a whole simulation: few columns, a long axis
        dict(name="ssm_probes", op="ssm", steps=8192, rows=3, cols=64, n=16, type="fp32", gate=False, starts=0.001, state=False),
        # a training window of a large mesh, several short trajectories in it
        dict(name="ssm_window_train", op="ssm_train", steps=20, rows=20011, cols=64, n=16, type="bf16", gate=True, starts=0.15, state=False),
        # a few probe rows of an odd width over a long trajectory, in training
        dict(name="ssm_probes_train", op="ssm_train", steps=2048, rows=5, cols=77, n=16, type="fp32", gate=False, starts=0.0, state=True),
        # the gradients of the 15-block network, tensor by tensor
        dict(name="clip_model", op="clip", sizes="model", layers=15, cols=128, rows=0, type="fp32", over=3.0),
        # a few large tables of embeddings or experts
        dict(name="clip_large", op="clip", sizes="even", layers=24, cols=0, rows=20000003, type="bf16", over=1.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["ln", "ln_grad", "conv", "conv_grad", "ssm", "ssm_train", "clip"])
    typ = rng.choice(["fp32", "bf16"])
    if op == "clip":
        if rng.random() < 0.5:
            return dict(op=op, sizes="model", layers=rng.randrange(1, 24), cols=rng.choice([32, 64, 128, 256]), rows=0, type=typ,
                        over=rng.choice([0.5, 1.1, 3.0, 100.0]))
        layers = _log(rng, 1, 300)
        return dict(op=op, sizes="even", layers=layers, cols=0, rows=_log(rng, 1, (1 << 27) // layers), type=typ,
                    over=rng.choice([0.5, 1.1, 3.0, 100.0]))
    cols = rng.choice([64, 128, 256]) if rng.random() < 0.5 else _log(rng, 1, 2048)
    if op in ("ln", "ln_grad"):
        c = dict(op=op, rows=_log(rng, 1, min(2000000, (1 << 27) // cols)), cols=cols, type=typ, res=rng.random() < 0.5)
        if op == "ln":
            c["out"] = rng.choice(["fp32", "bf16"])
        return c
    c = dict(op=op, type=typ, starts=rng.choice([0.0, 0.0, 0.02, 0.2]), state=rng.random() < 0.5)
    if op in ("conv", "conv_grad"):
        steps = 1 if rng.random() < 0.15 else _log(rng, 1, 8192)
        return dict(c, steps=steps, rows=_log(rng, 1, min(1000000, (1 << 26) // (steps * cols))), cols=cols,
                    width=rng.choice([1, 2, 3, 4, 4, 4, 6, 8]), silu=rng.random() < 0.7)
    cols = min(cols, 1024)
    n = 16 if rng.random() < 0.5 else rng.randrange(1, 65)
    steps = 1 if rng.random() < 0.15 else _log(rng, 1, 4096)
    most = (1 << 28 if op == "ssm" else 1 << 27) // n
    return dict(c, steps=steps, rows=_log(rng, 1, max(1, min(200000, most // (steps * cols)))), cols=cols, n=n,
                gate=rng.random() < 0.5)


def _tensors(c):
    """Lengths of a clip case's tensors."""
    if c["sizes"] == "even":
        return [max(1, c["rows"] - 7 * k) for k in range(c["layers"])]
    l = c["cols"]
    mlp = lambda fin, out: [fin * l, l, l * out, out]
    lengths = mlp(11, l) + [l, l] + mlp(4, l) + [l, l]
    lengths += (mlp(3 * l, l) + [l, l] + mlp(2 * l, l) + [l, l]) * c["layers"]
    return lengths + mlp(l, 5)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, f32 = DTYPE[c["type"]], torch.float32

    def normal(*shape, dtype=dt, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)

    s = dict(case=c)
    if c["op"] == "clip":
        # layers' gradients differ in size
        sizes = torch.exp(torch.randn(len(_tensors(c)), generator=torch.Generator().manual_seed(seed))).tolist()
        s["grads"] = [normal(m, scale=1e-2 * z) for m, z in zip(_tensors(c), sizes)]
        # the clipped ones lie one behind the other, as an update or an exchange wants them
        s["flat"] = torch.empty(sum(_tensors(c)), dtype=dt, device="cuda")
        s["outs"] = list(s["flat"].split(_tensors(c)))
        s["max_norm"] = 1e-2 * math.sqrt(sum(m * z * z for m, z in zip(_tensors(c), sizes))) / c["over"]
        s["norm"] = torch.empty(1, dtype=f32, device="cuda")
        s["list"] = None
        return s
    rows, cols = c["rows"], c["cols"]
    if c["op"] in ("ln", "ln_grad"):
        s["weight"], s["bias"] = 1 + normal(cols, dtype=f32, scale=0.1), normal(cols, dtype=f32, scale=0.1)
        # the residual stream's rows differ in size and offset, and some are zero
        size = torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))
        size[torch.rand(rows, 1, generator=gen, device="cuda") < 0.01] = 0
        s["x"] = ((torch.randn(rows, cols, generator=gen, device="cuda") + 0.5) * size).to(dt)
        s["res"] = normal(rows, cols) if c["res"] else None
        if c["op"] == "ln":
            s["total"] = torch.empty_like(s["x"]) if c["res"] else None
            s["y"] = torch.empty(rows, cols, dtype=DTYPE[c["out"]], device="cuda")
        else:
            s["dy"] = normal(rows, cols)
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty(cols, dtype=f32, device="cuda"), torch.empty(cols, dtype=f32, device="cuda")
        return s
    T = c["steps"]
    s["x"] = normal(T, rows, cols)
    s["starts"] = (torch.rand(T, generator=gen, device="cuda") < c["starts"]).to(torch.uint8) if c["starts"] else None
    if c["op"] in ("conv", "conv_grad"):
        W = c["width"]
        s["weight"], s["bias"] = normal(cols, W, dtype=f32, scale=W ** -0.5), normal(cols, dtype=f32, scale=0.1)
        s["past"] = normal(W - 1, rows, cols) if c["state"] else None
        if c["op"] == "conv":
            s["y"] = torch.empty_like(s["x"])
            s["past_out"] = torch.empty(W - 1, rows, cols, dtype=dt, device="cuda") if c["state"] else None
        else:
            s["dy"], s["dx"] = normal(T, rows, cols), torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
            s["d_past_out"] = normal(W - 1, rows, cols, dtype=f32) if c["state"] else None
            s["d_past"] = torch.empty(W - 1, rows, cols, dtype=f32, device="cuda") if c["state"] else None
        return s
    N = c["n"]
    s["dt"] = normal(T, rows, cols)
    # time constants from a few steps to some hundred
    s["dt_bias"] = -1.0 - 4.0 * torch.rand(cols, generator=gen, device="cuda")
    s["A"] = -torch.arange(1, N + 1, device="cuda", dtype=f32) * torch.exp(normal(cols, N, dtype=f32, scale=0.1))
    s["B"], s["C"] = normal(T, rows, N), normal(T, rows, N)
    s["D"] = 1 + normal(cols, dtype=f32, scale=0.1)
    s["z"] = normal(T, rows, cols) if c["gate"] else None
    s["h0"] = normal(rows, cols, N, dtype=f32) if c["state"] else None
    s["h_last"] = torch.empty(rows, cols, N, dtype=f32, device="cuda") if c["state"] else None
    s["y"] = torch.empty_like(s["x"])
    if c["op"] == "ssm_train":
        s["dy"] = normal(T, rows, cols)
        s["dh_last"] = normal(rows, cols, N, dtype=f32) if c["state"] else None
        s["dx"], s["ddt"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["dz"] = torch.empty_like(s["x"]) if c["gate"] else None
        s["dB"], s["dC"] = torch.empty_like(s["B"]), torch.empty_like(s["C"])
        s["dA"], s["dD"], s["dbias"] = torch.empty_like(s["A"]), torch.empty_like(s["D"]), torch.empty_like(s["D"])
        s["dh0"] = torch.empty_like(s["h0"]) if c["state"] else None
    return s


# ------------------------------------------------------------- plain forms ---
def _ln(s):
    t = s["x"].float()
    if s["res"] is not None:
        t = t + s["res"].float()
    d = t - t.mean(1, keepdim=True)
    y = d * torch.rsqrt((d * d).mean(1, keepdim=True) + EPS) * s["weight"] + s["bias"]
    return (y.to(s["y"].dtype), t.to(s["x"].dtype)) if s["res"] is not None else (y.to(s["y"].dtype),)


def _ln_grad(s):
    t, dy = s["x"].float(), s["dy"].float()
    d = t - t.mean(1, keepdim=True)
    inv = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    u, g = d * inv, s["weight"] * dy
    dx = inv * (g - g.mean(1, keepdim=True) - u * (g * u).mean(1, keepdim=True))
    if s["res"] is not None:
        dx = dx + s["res"].float()
    return dx.to(s["dx"].dtype), (dy * u).sum(0, dtype=torch.float64).float(), dy.sum(0, dtype=torch.float64).float()


def _lags(s):
    """Whether step t sees the step k before it, [T][W] by lag k: no start lies between."""
    T, W = s["x"].shape[0], s["case"]["width"]
    part = torch.zeros(T, dtype=torch.int64, device="cuda") if s["starts"] is None else s["starts"].long().cumsum(0)
    part = torch.cat([part.new_zeros(W - 1), part])  # what came before is of the first part
    return part.unfold(0, W, 1).flip(1) == part[W - 1:, None]


def _before(s):
    """The inputs with the W - 1 before them, float32."""
    x, W = s["x"].float(), s["case"]["width"]
    past = s["past"].float() if s["past"] is not None else x.new_zeros(W - 1, *x.shape[1:])
    return torch.cat([past, x])


def _pre(s, xp, sees):
    """bias + the weighted inputs: windows [T][rows][cols][W], newest first."""
    W = s["case"]["width"]
    win = xp.unfold(0, W, 1).flip(3) * sees[:, None, None, :].float()
    return win, (win * s["weight"].flip(1)).sum(3) + s["bias"]


def _conv(s):
    xp, sees, W = _before(s), _lags(s), s["case"]["width"]
    y = _pre(s, xp, sees)[1]
    if s["case"]["silu"]:
        y = y * torch.sigmoid(y)
    if s["past"] is None:
        return (y.to(s["x"].dtype),)
    part = torch.zeros(W - 1 + s["x"].shape[0], dtype=torch.int64, device="cuda")
    if s["starts"] is not None:
        part[W - 1:] = s["starts"].long().cumsum(0)
    left = xp * (part == part[-1])[:, None, None].float() if s["starts"] is not None else xp
    return y.to(s["x"].dtype), left[xp.shape[0] - (W - 1):].to(s["x"].dtype)


def _conv_grad(s):
    xp, sees, W = _before(s), _lags(s), s["case"]["width"]
    win, v = _pre(s, xp, sees)
    d = s["dy"].float()
    if s["case"]["silu"]:
        g = torch.sigmoid(v)
        d = d * (g * (1 + v * (1 - g)))
    dw = (d[..., None] * win).sum((0, 1), dtype=torch.float64).float().flip(1)
    # input i (from the oldest past one on) goes to the steps i - (W - 1) + k, k = 0 .. W - 1
    pad = torch.cat([d.new_zeros(W - 1, *d.shape[1:]), d, d.new_zeros(W - 1, *d.shape[1:])]).unfold(0, W, 1)
    m = torch.cat([sees.new_zeros(W - 1, W), sees, sees.new_zeros(W - 1, W)]).unfold(0, W, 1).diagonal(dim1=1, dim2=2)
    dxp = (pad * m[:, None, None, :].float() * s["weight"].flip(1)).sum(3)
    if s["past"] is not None:
        T = s["x"].shape[0]
        part = torch.zeros(W - 1 + T, dtype=torch.int64, device="cuda")
        if s["starts"] is not None:
            part[W - 1:] = s["starts"].long().cumsum(0)
        dxp[T:] += s["d_past_out"] * (part == part[-1])[T:, None, None].float()
    dx, db = dxp[W - 1:].to(s["x"].dtype), d.sum((0, 1), dtype=torch.float64).float()
    return (dx, dw, db) if s["past"] is None else (dx, dw, db, dxp[:W - 1])


def _linear(f, b):
    """h_t = f_t h_{t-1} + b_t along the first axis from h = 0: pairs (f, b) joined over 1, 2, 4, ... steps."""
    d = 1
    while d < f.shape[0]:
        b = torch.cat([b[:d], b[d:] + f[d:] * b[:-d]])
        f = torch.cat([f[:d], f[d:] * f[:-d]])
        d *= 2
    return b


def _ssm_parts(s):
    """delta, its argument, exp(delta A) (0 at a start) and every state, float32."""
    v = s["dt"].float() + s["dt_bias"]
    delta = v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    f = torch.exp(delta[..., None] * s["A"])
    if s["starts"] is not None:
        f = f * (s["starts"] == 0).float()[:, None, None, None]
    b = (delta * s["x"].float())[..., None] * s["B"].float()[:, :, None, :]
    if s["h0"] is not None:
        b[0] += f[0] * s["h0"]
    return delta, v, f, _linear(f, b)


def _ssm_out(s, h):
    y = (h * s["C"].float()[:, :, None, :]).sum(3) + s["D"] * s["x"].float()
    return y


def _ssm(s):
    h = _ssm_parts(s)[3]
    y = _ssm_out(s, h)
    if s["z"] is not None:
        z = s["z"].float()
        y = y * (z * torch.sigmoid(z))
    y = y.to(s["x"].dtype)
    return (y,) if s["h0"] is None else (y, h[-1].clone())


def _ssm_train(s):
    delta, v, f, h = _ssm_parts(s)
    x, B, C, dy, dt = s["x"].float(), s["B"].float(), s["C"].float(), s["dy"].float(), s["x"].dtype
    o = _ssm_out(s, h)
    y, dz = o, None
    if s["z"] is not None:
        z = s["z"].float()
        g = torch.sigmoid(z)
        y, dz, dy = o * (z * g), (dy * o * (g * (1 + z * (1 - g)))).to(dt), dy * (z * g)
    y, last = y.to(dt), h[-1].clone()
    d = dy[..., None] * C[:, :, None, :]
    if s["dh_last"] is not None:
        d[-1] += s["dh_last"]
    G = _linear(torch.cat([f[1:], torch.zeros_like(f[:1])]).flip(0), d.flip(0)).flip(0)  # gradient of every state
    del d
    dC = (dy[..., None] * h).sum(2)
    dB = ((delta * x)[..., None] * G).sum(2)
    GB = (G * B[:, :, None, :]).sum(3)
    prev = torch.cat([(s["h0"] if s["h0"] is not None else torch.zeros_like(h[0]))[None], h[:-1]])
    del h
    dh0 = f[0] * G[0] if s["h0"] is not None else None
    G = G * f * prev
    del f, prev
    ddelta = (G * s["A"]).sum(3) + GB * x
    dA = (G * delta[..., None]).sum((0, 1), dtype=torch.float64).float()
    dv = ddelta * torch.sigmoid(v)
    dx = GB * delta + s["D"] * dy
    dD, dbias = (dy * x).sum((0, 1), dtype=torch.float64).float(), dv.sum((0, 1), dtype=torch.float64).float()
    out = dict(y=y, dx=dx.to(dt), ddt=dv.to(dt), dz=dz, dA=dA, dB=dB.to(dt), dC=dC.to(dt), dD=dD, dbias=dbias)
    if s["h0"] is not None:
        out.update(h_last=last, dh0=dh0)
    return out


def _clip(s):
    norm = torch.sqrt(torch.stack([(g.float() * g.float()).sum(dtype=torch.float64) for g in s["grads"]]).sum()).float()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    for g, out in zip(s["grads"], s["outs"]):
        out.copy_(g.float() * factor)
    return norm[None], s["flat"]


# --------------------------------------------------------------------- run ---
def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"ln": _ln, "ln_grad": _ln_grad, "conv": _conv, "conv_grad": _conv_grad, "ssm": _ssm, "ssm_train": _ssm_train,
                "clip": _clip}[op](s)
    import paper_2307_13592_amd as mgn
    if op == "ln":
        mgn.mgn_layer_norm(s["x"], s["weight"], s["bias"], s["y"], res=s["res"], total=s["total"], eps=EPS)
        return (s["y"], s["total"]) if s["res"] is not None else (s["y"],)
    if op == "ln_grad":
        mgn.mgn_layer_norm_grad(s["x"], s["weight"], s["dy"], s["dx"], s["dweight"], s["dbias"], d_total=s["res"], eps=EPS)
        return s["dx"], s["dweight"], s["dbias"]
    if op == "conv":
        mgn.mgn_causal_conv(s["x"], s["weight"], s["y"], bias=s["bias"], past=s["past"], past_out=s["past_out"],
                            starts=s["starts"], silu=s["case"]["silu"])
        return (s["y"],) if s["past"] is None else (s["y"], s["past_out"])
    if op == "conv_grad":
        mgn.mgn_causal_conv_grad(s["x"], s["weight"], s["dy"], s["dx"], s["dweight"], s["dbias"], bias=s["bias"], past=s["past"],
                                 d_past=s["d_past"], d_past_out=s["d_past_out"], starts=s["starts"], silu=s["case"]["silu"])
        return (s["dx"], s["dweight"], s["dbias"]) if s["past"] is None else (s["dx"], s["dweight"], s["dbias"], s["d_past"])
    if op == "clip":
        if s["list"] is None:  # a training program makes it once for its gradients
            s["list"] = mgn.mgn_grad_list(s["grads"], s["outs"])
        mgn.mgn_grad_clip(s["list"], s["max_norm"], s["norm"])
        return s["norm"], s["flat"]
    args = dict(D=s["D"], dt_bias=s["dt_bias"], z=s["z"], starts=s["starts"], softplus=True)
    if op == "ssm":
        mgn.mgn_selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["y"], h0=s["h0"], h_last=s["h_last"], **args)
        return (s["y"],) if s["h0"] is None else (s["y"], s["h_last"])
    marks = mgn.mgn_selective_marks(s["x"], s["A"])
    mgn.mgn_selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["y"], h0=s["h0"], h_last=s["h_last"], marks=marks, **args)
    mgn.mgn_selective_scan_grad(s["x"], s["dt"], s["A"], s["B"], s["C"], marks, s["dy"], s["dx"], s["ddt"], s["dA"], s["dB"],
                                s["dC"], dD=s["dD"], d_bias=s["dbias"], dz=s["dz"], dh_last=s["dh_last"], dh0=s["dh0"], **args)
    out = {k: s[k] for k in ("y", "dx", "ddt", "dz", "dA", "dB", "dC", "dD", "dbias")}
    if s["h0"] is not None:
        out.update(h_last=s["h_last"], dh0=s["dh0"])
    return out


def work(case):
    c, size = case, {"fp32": 4, "bf16": 2}
    b = size[c["type"]]
    if c["op"] == "clip":
        m = sum(_tensors(c))
        return {"bytes": 2 * b * m + 4, "flops": 3 * m}
    cols = c["cols"]
    if c["op"] == "ln":
        m = c["rows"] * cols
        return {"bytes": m * (b * (3 if c["res"] else 1) + size[c["out"]]) + 8 * cols, "flops": 8 * m}
    if c["op"] == "ln_grad":
        m = c["rows"] * cols
        return {"bytes": m * b * (4 if c["res"] else 3) + 12 * cols, "flops": 15 * m}
    T, m = c["steps"], c["steps"] * c["rows"] * cols
    one = c["rows"] * cols
    if c["op"] in ("conv", "conv_grad"):
        W = c["width"]
        act = 5 if c["silu"] else 0
        if c["op"] == "conv":
            return {"bytes": 2 * b * m + (2 * b * (W - 1) * one if c["state"] else 0) + 4 * cols * (W + 1), "flops": m * (2 * W + act)}
        return {"bytes": 3 * b * m + ((b + 8) * (W - 1) * one if c["state"] else 0) + 8 * cols * (W + 1),
                "flops": m * (6 * W + 2 * act + 1)}
    N, gate = c["n"], 1 if c["gate"] else 0
    pair = 2 * b * T * c["rows"] * N
    fwd = {"bytes": m * b * (3 + gate) + pair + 4 * cols * (N + 2) + (8 * one * N if c["state"] else 0), "flops": m * (7 * N + 10)}
    if c["op"] == "ssm":
        return fwd
    # x, dt, dy, z read, y, dx, ddt, dz written; B, C and their gradients
    return {"bytes": m * b * (6 + 2 * gate) + 2 * pair + 8 * cols * (N + 2) + (16 * one * N if c["state"] else 0),
            "flops": m * (21 * N + 40)}


# ------------------------------------------------------------------- exact ---
def exact(case, seed):
    """run()'s outputs from the definitions in 64 bits."""
    s, c = prepare(case, seed), case
    f64 = torch.float64
    if c["op"] == "clip":
        total = sum(float(torch.dot(g.to(f64), g.to(f64))) for g in s["grads"])
        norm = math.sqrt(total)
        k = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
        return torch.tensor([norm], dtype=f64, device="cuda"), torch.cat([g.to(f64) * k for g in s["grads"]])
    if c["op"] in ("ln", "ln_grad"):
        n = c["cols"]
        t = s["x"].to(f64)
        if c["op"] == "ln" and s["res"] is not None:
            t += s["res"].to(f64)
        mean = t.sum(1, keepdim=True) / n
        dev = torch.sqrt(((t - mean) ** 2).sum(1, keepdim=True) / n + EPS)
        u = (t - mean) / dev
        if c["op"] == "ln":
            y = u * s["weight"].to(f64) + s["bias"].to(f64)
            return (y, t) if s["res"] is not None else (y,)
        dy = s["dy"].to(f64)
        g = dy * s["weight"].to(f64)
        # (t - mean) / dev: the gradient less its parts along 1 and along u
        dx = (g - g.sum(1, keepdim=True) / n - u * ((g * u).sum(1, keepdim=True) / n)) / dev
        if s["res"] is not None:
            dx += s["res"].to(f64)
        return dx, (dy * u).sum(0), dy.sum(0)
    T, rows, cols = c["steps"], c["rows"], c["cols"]
    fresh = s["starts"].tolist() if s["starts"] is not None else [0] * T
    x = s["x"].to(f64)
    if c["op"] in ("conv", "conv_grad"):
        W = c["width"]
        w, bias = s["weight"].to(f64), s["bias"].to(f64)
        zero = torch.zeros(rows, cols, dtype=f64, device="cuda")
        line = [(s["past"][k].to(f64) if s["past"] is not None else zero) for k in range(W - 1)]  # inputs that the next step sees
        grads = c["op"] == "conv_grad"
        y, seen, at = torch.empty(T, rows, cols, dtype=f64, device="cuda"), [], list(range(-(W - 1), 0))
        for t in range(T):
            if fresh[t]:
                at = [None] * (W - 1)
            now = at + [t]
            y[t] = bias
            for k in range(W):
                if now[k] is not None:
                    v = x[now[k]] if now[k] >= 0 else line[now[k] + W - 1]
                    y[t] += w[:, k] * v
            seen.append(now)
            at = now[1:]
        value = lambda i: x[i] if i >= 0 else line[i + W - 1]
        if not grads:
            out = y / (1 + torch.exp(-y)) if c["silu"] else y
            if s["past"] is None:
                return (out,)
            left = [zero if i is None else value(i) for i in at]
            return out, torch.stack(left) if left else zero[None][:0]
        dz = s["dy"].to(f64)
        if c["silu"]:
            e = torch.exp(-y)
            dz = dz * (1 / (1 + e) + y * e / (1 + e) ** 2)
        dw, dxp = torch.zeros(cols, W, dtype=f64, device="cuda"), torch.zeros(T + W - 1, rows, cols, dtype=f64, device="cuda")
        for t in range(T):
            for k in range(W):
                i = seen[t][k]
                if i is not None:
                    dw[:, k] += (dz[t] * value(i)).sum(0)
                    dxp[i + W - 1] += w[:, k] * dz[t]
        if s["past"] is None:
            return dxp[W - 1:], dw, dz.sum((0, 1))
        for k, i in enumerate(at):
            if i is not None:
                dxp[i + W - 1] += s["d_past_out"][k].to(f64)
        return dxp[W - 1:], dw, dz.sum((0, 1)), dxp[:W - 1]
    N = c["n"]
    A, D, bias = s["A"].to(f64), s["D"].to(f64), s["dt_bias"].to(f64)
    B, C, dt = s["B"].to(f64), s["C"].to(f64), s["dt"].to(f64) + bias
    delta = torch.where(dt > 0, dt, torch.zeros_like(dt)) + torch.log1p(torch.exp(-dt.abs()))
    zero = torch.zeros(rows, cols, N, dtype=f64, device="cuda")
    h0 = s["h0"].to(f64) if s["h0"] is not None else zero
    train = c["op"] == "ssm_train"
    h, hist, o = h0, [], torch.empty(T, rows, cols, dtype=f64, device="cuda")
    for t in range(T):
        before = zero if fresh[t] else h
        h = torch.exp(delta[t, :, :, None] * A) * before + (delta[t] * x[t])[:, :, None] * B[t][:, None, :]
        o[t] = (h * C[t][:, None, :]).sum(2) + D * x[t]
        if train:
            hist.append(h)
    sz = None
    if s["z"] is not None:
        z = s["z"].to(f64)
        sg = 1 / (1 + torch.exp(-z))
        sz = z * sg
    y = o * sz if sz is not None else o
    if not train:
        return (y,) if s["h0"] is None else (y, h)
    dy = s["dy"].to(f64)
    dz = None
    if sz is not None:
        dz = dy * o * (sg + sz * (1 - sg))
        dy = dy * sz
    dx, ddt, dB, dC = torch.empty_like(x), torch.empty_like(x), torch.empty_like(B), torch.empty_like(C)
    dA = torch.zeros_like(A)
    G = s["dh_last"].to(f64) if s["dh_last"] is not None else zero
    for t in range(T - 1, -1, -1):
        G = G + dy[t][:, :, None] * C[t][:, None, :]
        before = zero if fresh[t] else (hist[t - 1] if t else h0)
        f = torch.exp(delta[t, :, :, None] * A)
        dC[t] = (dy[t][:, :, None] * hist[t]).sum(1)
        dB[t] = (G * (delta[t] * x[t])[:, :, None]).sum(1)
        inner = (G * B[t][:, None, :]).sum(2)
        dx[t] = inner * delta[t] + D * dy[t]
        through = G * f * before
        ddt[t] = ((through * A).sum(2) + inner * x[t]) / (1 + torch.exp(-dt[t]))
        dA += (through * delta[t][:, :, None]).sum(0)
        G = zero if fresh[t] else G * f
    out = dict(y=y, dx=dx, ddt=ddt, dz=dz, dA=dA, dB=dB, dC=dC, dD=(dy * x).sum((0, 1)), dbias=ddt.sum((0, 1)))
    if s["h0"] is not None:
        out.update(h_last=hist[-1], dh0=G)
    return out
