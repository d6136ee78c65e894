"""A refused clipped update leaves the gradient and the parameters as they were."""
import numpy as np
import pytest
import torch

import paper_2307_13592_amd as mgn
import synth
from paper_2307_13592_amd.lockstep import Lockstep
from paper_2307_13592_amd.runner import Session

pytestmark = pytest.mark.gpu
K, L, D = 1, 64, 2


def _parts(P):
    mesh = synth.sector(4, 8, 6, 4, seed=3)
    part = mgn.mgn_partition_slabs(mesh.key, P)
    graphs = [mgn.mgn_graph_build(mesh.send, mesh.recv, part, mesh.n_nodes, p) for p in range(P)]
    nf, ef = synth.node_features(mesh, 3), synth.edge_features(mesh)
    params = synth.init_params(synth.param_shapes(L, K, D), 3)
    return part, graphs, [nf[g["l2g"][:g["n_owned"]]] for g in graphs], [ef[g["eperm"]] for g in graphs], params


def _unchanged(model, grad, calls):
    before, params = grad.clone(), mgn.mgn_get_params(model)
    for call in calls:
        with pytest.raises((ValueError, mgn.MgnError)):
            call()
        assert torch.equal(grad, before) and np.array_equal(mgn.mgn_get_params(model), params)


def test_session():
    _, (g,), (nf,), (ef,), params = _parts(1)
    s = Session(L, K, D, "fp32", g, nf, ef, np.zeros((K, 0, L), np.float32), params)
    n = s.n_params
    s.d_params.normal_()
    _unchanged(s.model, s.d_params, [lambda: s.sgd(float("nan"), max_norm=1.0), lambda: s.sgd(1e39, max_norm=1.0),
                                     lambda: s.sgd(0.1, max_norm=0.0), lambda: s.sgd(0.1, max_norm=float("inf"))])
    for grad in (torch.ones(n, dtype=torch.bfloat16, device="cuda"), torch.ones(n, dtype=torch.float64, device="cuda"),
                 torch.ones(n + 1, device="cuda"), torch.ones(n, 2, device="cuda")[:, 0]):
        _unchanged(s.model, grad, [lambda: s.sgd(0.1, grad, max_norm=1.0), lambda: s.sgd(0.1, grad)])
    s.close()


def test_parts_in_lockstep():
    part, graphs, nfs, efs, params = _parts(2)
    ls = Lockstep(L, K, D, "fp32", part, graphs, nfs, efs, params)
    ls.d_params.normal_()
    for s in ls.sessions:
        _unchanged(s.model, ls.d_params, [lambda: ls.sgd(float("nan"), max_norm=1.0), lambda: ls.sgd(0.1, max_norm=-1.0)])
    ls.close()
