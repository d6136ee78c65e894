"""Device-side session for one partition: uploads a host-built local graph and
its inputs to HBM once, then runs the training step through the C ABI.
Argument marshalling only; the step itself runs in libmgn's kernels."""
from __future__ import annotations

import numpy as np
import torch

from . import (MGN_BF16, MGN_FP32, graph_struct, mgn_backward, mgn_create, mgn_destroy, mgn_forward,
               mgn_graph_validate, mgn_mse_grad, mgn_param_count, mgn_set_params, mgn_set_recompute,
               mgn_norm_accumulate, mgn_norm_apply, MGN_NORM_WORK_PER_COL, mgn_rollout_update, mgn_set_h1_stash,
               mgn_set_inference, mgn_sgd_step, mgn_workspace_size, mgn_gated_scan, mgn_gated_scan_grad, mgn_rms_norm,
               mgn_rms_norm_grad, mgn_rows_load8, mgn_rows_store8, rows8_blocks, _on)


class Session:
    def __init__(self, latent: int, K: int, depth: int, precision: str, graph: dict, node_feat, edge_feat, halo,
                 params, device: str = "cuda", node_in: int = 11, edge_in: int = 4, node_out: int = 5,
                 recompute: int = 0, chunk_edges: int = 0, inference: bool = False, h1_stash: int = 0):
        """recompute: edge-stream checkpoint interval (mgn_set_recompute, bf16;
        0: keep every block); -1: the smallest interval whose workspace fits
        the device's free memory with 8 GiB to spare.  h1_stash: blocks whose
        first-Linear ReLU output the forward keeps for the backward
        (row-split kernels, mgn_set_h1_stash); -1: as many as the device's
        free memory holds beside the rest of the workspace (with 8 GiB to
        spare)."""
        if not torch.cuda.is_available():
            raise RuntimeError("libmgn needs a HIP device")
        self.device = torch.device(device)
        self.K, self.latent = K, latent
        prec = MGN_BF16 if precision == "bf16" else MGN_FP32
        self.model = mgn_create(latent, K, depth, prec, node_in, edge_in, node_out)
        dev = lambda a, dt: torch.as_tensor(np.ascontiguousarray(a, dtype=dt)).to(self.device)
        self.g = dict(n_owned=int(graph["n_owned"]), n_halo=int(graph["n_halo"]), n_edges=int(graph["n_edges"]),
                      row_ptr=dev(graph["row_ptr"], np.int32), send=dev(graph["send"], np.int32),
                      trow_ptr=dev(graph["trow_ptr"], np.int32), tedge=dev(graph["tedge"], np.int32))
        self.gs = graph_struct(self.g)
        no, nh, ne = self.g["n_owned"], self.g["n_halo"], self.g["n_edges"]
        self.node_feat = dev(np.asarray(node_feat).reshape(no, node_in), np.float32)
        self.edge_feat = dev(np.asarray(edge_feat).reshape(ne, edge_in), np.float32)
        self.halo = dev(halo, np.float32) if (nh > 0 and K > 0) else None
        self.n_params = mgn_param_count(self.model)
        self.set_params(params)
        mgn_graph_validate(self.model, self.gs)
        if recompute < 0 and not inference and K > 0 and ne > 0:
            # the smallest checkpoint interval whose workspace (as the library
            # plans it) leaves 8 GiB of the free memory: fewer blocks'
            # edge forwards repeated in the backward
            free = torch.cuda.mem_get_info(self.device)[0]
            for s in range(1, K + 1):
                mgn_set_recompute(self.model, s, chunk_edges)
                if mgn_workspace_size(self.model, self.gs) + (8 << 30) <= free:
                    recompute = s
                    break
            else:
                recompute = K
        self.recompute = max(recompute, 0)
        if self.recompute:
            mgn_set_recompute(self.model, self.recompute, chunk_edges)
        if inference:
            mgn_set_inference(self.model, True)
        self.ws_bytes = mgn_workspace_size(self.model, self.gs)
        if h1_stash < 0 and not inference and K > 0 and ne > 0:
            # the most blocks whose workspace (as the library plans it) leaves
            # 8 GiB of the free memory
            free = torch.cuda.mem_get_info(self.device)[0]
            h1_stash = 0
            for n in range(K, 0, -1):
                mgn_set_h1_stash(self.model, n)
                if mgn_workspace_size(self.model, self.gs) + (8 << 30) <= free:
                    h1_stash = n
                    break
        self.h1_stash = max(h1_stash, 0)
        mgn_set_h1_stash(self.model, self.h1_stash)
        self.ws_bytes = mgn_workspace_size(self.model, self.gs)
        self.workspace = torch.empty(max(self.ws_bytes, 256), dtype=torch.uint8, device=self.device)
        self.out = torch.empty((no, node_out), dtype=torch.float32, device=self.device)
        self.d_params = None if inference else torch.empty(self.n_params, dtype=torch.float32, device=self.device)
        self.d_halo = (torch.empty((K, nh, latent), dtype=torch.float32, device=self.device)
                       if (nh and K and not inference) else None)

    def set_params(self, params):
        if isinstance(params, torch.Tensor):
            mgn_set_params(self.model, params.to(self.device, torch.float32).contiguous())
        else:
            mgn_set_params(self.model, np.asarray(params, np.float32))

    def forward(self, stream=None):
        mgn_forward(self.model, self.gs, self.node_feat, self.edge_feat, self.halo, self.out, self.workspace, stream)
        return self.out

    def backward(self, d_out, accumulate: bool = False, stream=None):
        with _on(stream, self.device):
            if not isinstance(d_out, torch.Tensor):
                d_out = torch.as_tensor(np.ascontiguousarray(d_out, np.float32)).to(self.device)
            d_out = d_out.contiguous()
        mgn_backward(self.model, d_out, self.d_params, accumulate, self.d_halo, stream)
        return self.d_params, self.d_halo

    def sgd(self, lr: float, grad=None, stream=None):
        """Parameter update with the last backward's gradient (or `grad`)."""
        mgn_sgd_step(self.model, self.d_params if grad is None else grad, lr, stream)

    def rollout(self, steps: int, col0: int = 3, stream=None, memory=None, history=None):
        """`steps` next-step predictions, each fed back into the flow columns
        of the node features (q <- q + p); returns the outputs of every step.
        memory: a GatedMemory of this session's outputs with a gate; the
        increments fed back are then its states, h <- f h + (1 - f) p.
        history: a LatentCache of at least steps * n_owned slots; the outputs
        are then kept there in 8 bits (step t in slots t n_owned ..), and the
        cache is returned.  (A row of a few columns has a scale of 4 bytes of its
        own: five columns take 9 bytes, against 20 in float32 and 10 in bfloat16.)"""
        n = self.out.shape[0]
        outs = []
        if history is not None and (history.cols != self.out.shape[1] or history.slots < steps * n):
            raise ValueError("history: expected steps * n_owned slots of node_out columns")
        for t in range(steps):
            self.forward(stream)
            if history is not None:
                history.store(self.out, first=t * n, stream=stream)
            else:
                with _on(stream, self.device):
                    outs.append(self.out.clone())
            p = self.out if memory is None else memory.step(self.out, stream=stream)
            mgn_rollout_update(p, self.node_feat, col0, stream)
        return outs if history is None else history

    def mse(self, target, mask=None, stream=None):
        with _on(stream, self.device):
            loss = torch.empty(2, dtype=torch.float32, device=self.device)
            d_out = torch.empty_like(self.out)
        mgn_mse_grad(self.out, target, mask, loss, d_out, stream)
        return loss, d_out

    def close(self):
        """Destroys the model and drops every device buffer of the session."""
        if getattr(self, "model", None):
            mgn_destroy(self.model)
            self.model = None
        for k in ("workspace", "out", "d_params", "d_halo", "node_feat", "edge_feat", "halo", "g"):
            setattr(self, k, None)
        torch.cuda.empty_cache()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Normalizer:
    """Running per-column statistics of one kind of input (increments, node
    features or edge features) on the device, for Normalize of Algorithm 1:
    accumulate() adds rows while training, apply() standardises."""

    def __init__(self, cols: int, device: str = "cuda", eps: float = 1e-8):
        self.cols, self.eps = cols, eps
        self.stats = torch.zeros(1 + 2 * cols, dtype=torch.float64, device=device)
        self.work = torch.empty(MGN_NORM_WORK_PER_COL * cols, dtype=torch.float64, device=device)

    def accumulate(self, x, stream=None):
        mgn_norm_accumulate(x, self.stats, self.work, stream)

    def apply(self, x, out=None, stream=None):
        with _on(stream, x.device):
            out = torch.empty_like(x) if out is None else out
        mgn_norm_apply(x, self.stats, out, self.eps, stream)
        return out


class LatentCache:
    """`slots` rows of `cols` columns held in 8 bits on the device (codes q,
    one scale per 128 columns, cols + 4 ceil(cols / 128) bytes a row): packed halo
    rows, or the history of a rollout or of a trajectory's node latents."""

    def __init__(self, slots: int, cols: int, device: str = "cuda"):
        self.slots, self.cols = slots, cols
        self.q = torch.zeros((slots, cols), dtype=torch.uint8, device=device)
        self.scale = torch.ones((slots, rows8_blocks(cols)), dtype=torch.float32, device=device)

    def store(self, src, first: int = 0, src_rows=None, slots=None, stream=None):
        """Rows of src (or its src_rows) into the slots given, or into first,
        first + 1, ..."""
        if slots is not None:
            mgn_rows_store8(src, self.q, self.scale, src_rows, slots, stream)
            return
        q, scale = self._span(first, src.shape[0] if src_rows is None else src_rows.numel())
        mgn_rows_store8(src, q, scale, src_rows, None, stream)

    def load(self, dst, first: int = 0, slots=None, dst_rows=None, add: bool = False, stream=None):
        """The slots given, or first, first + 1, ..., into dst (or its dst_rows)."""
        if slots is not None:
            mgn_rows_load8(self.q, self.scale, dst, slots, dst_rows, add, stream)
        else:
            q, scale = self._span(first, dst.shape[0] if dst_rows is None else dst_rows.numel())
            mgn_rows_load8(q, scale, dst, None, dst_rows, add, stream)
        return dst

    def window(self, first: int, steps: int, rows: int):
        """Codes and scales of steps x rows slots from `first` on, as the
        recurrence reads them: ([steps][rows][cols], [steps][rows][blocks])."""
        q, scale = self._span(first, steps * rows)
        return q.view(steps, rows, self.cols), scale.view(steps, rows, -1)

    def _span(self, first: int, n: int):
        if first < 0 or first + n > self.slots:
            raise ValueError(f"slots {first} .. {first + n} of {self.slots}")
        return self.q[first:first + n], self.scale[first:first + n]


class RmsNorm:
    """Root-mean-square norm of node rows with a weight per column, and the
    addition of a residual before it."""

    def __init__(self, cols: int, device: str = "cuda", eps: float = 1e-6):
        self.cols, self.eps = cols, eps
        self.weight = torch.ones(cols, dtype=torch.float32, device=device)
        self.d_weight = torch.zeros_like(self.weight)

    def apply(self, x, res=None, dtype=None, stream=None):
        """(y, t): y the norm of t = x + res (of x without a residual) in
        `dtype` (x's by default)."""
        with _on(stream, x.device):
            y = torch.empty_like(x, dtype=x.dtype if dtype is None else dtype)
            total = x if res is None else torch.empty_like(x)
        mgn_rms_norm(x, self.weight, y, res, None if res is None else total, None, self.eps, stream)
        return y, total

    def store(self, x, cache: LatentCache, first: int = 0, res=None, stream=None):
        """The norm of x + res in 8 bits, into the cache's slots from `first`
        on; returns the sum."""
        q, scale = cache._span(first, x.shape[0])
        with _on(stream, x.device):
            total = x if res is None else torch.empty_like(x)
        mgn_rms_norm(x, self.weight, q, res, None if res is None else total, scale, self.eps, stream)
        return total

    def grad(self, total, dy, d_total=None, accumulate: bool = False, stream=None):
        """dL/dt from dy and the gradient that reaches t otherwise; d_weight
        takes (accumulate: adds) dL/dweight."""
        with _on(stream, total.device):
            dx = torch.empty_like(total)
        mgn_rms_norm_grad(total, self.weight, dy, dx, self.d_weight, d_total, accumulate, None, self.eps, stream)
        return dx


class GatedMemory:
    """A gated linear recurrence over time on rows of `cols` columns:
    h <- f h + (1 - f) x with f = sigmoid(g).  step() carries `state` along a
    rollout; scan() and grad() run whole trajectories.  gate: logits
    [rows][cols] that step() uses when it is given none."""

    def __init__(self, rows: int, cols: int, device: str = "cuda", gate=None):
        self.state = torch.zeros((rows, cols), dtype=torch.float32, device=device)
        self.h0 = torch.zeros_like(self.state)  # the state that the last scan() began with
        self.gate = gate

    def step(self, x, g=None, x_scale=None, stream=None):
        """One time step (x, g [rows][cols]); returns the state."""
        g = self.gate if g is None else g
        if g is None:
            raise ValueError("g: no gate given")
        mgn_gated_scan(g[None], x[None], None, self.state, self.state, None,
                       None if x_scale is None else x_scale[None], None, stream)
        return self.state

    def scan(self, g, x, starts=None, x_scale=None, stream=None):
        """Every state h of a trajectory [steps][rows][cols] that continues from
        `state`, which becomes the last one; h.h0 is the state it began with."""
        with _on(stream, g.device):
            h = torch.empty(g.shape, dtype=torch.float32, device=g.device)
            h0 = torch.empty_like(self.state)
        none = None if x_scale is None else x_scale[:0]
        mgn_gated_scan(g[:0], x[:0], None, h0, self.state, None, none, None, stream)  # h0 <- state
        mgn_gated_scan(g, x, h, self.state, h0, starts, x_scale, None, stream)
        self.h0 = h.h0 = h0
        return h

    def grad(self, g, x, h, dh=None, dh_last=None, starts=None, x_scale=None, stream=None, h0=None):
        """(dg, dx, dh0) of the scan() that returned h.  h0: the state which that
        began with; without it h.h0, and for an h that carries none (a copy) that
        of the last scan()."""
        with _on(stream, g.device):
            dg, dx = torch.empty_like(g), torch.empty_like(g)
            dh0 = torch.empty_like(self.state)
        h0 = getattr(h, "h0", self.h0) if h0 is None else h0
        mgn_gated_scan_grad(g, x, h, dg, dx, dh, dh_last, dh0, h0, starts, x_scale, None, stream)
        return dg, dx, dh0
