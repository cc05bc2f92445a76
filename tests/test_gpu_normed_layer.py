"""One layer in training (runner.NormedLayer): layer norm with its 8-bit checkpoint, a product with
binarized weights, the aggregation, and every gradient from the checkpoint, against 64-bit formulas
over a dense adjacency, and against differences of the loss."""
import numpy as np
import pytest
import torch

import norm_reference as R
from gpu_helpers import to_dev
from paper_2010_07565_gb300 import binding as B
from paper_2010_07565_gb300 import inputs
from paper_2010_07565_gb300.runner import NormedLayer

pytestmark = pytest.mark.gpu


def dense(rowptr, colidx):
    N = len(rowptr) - 1
    A = np.eye(N)
    for i in range(N):
        for j in colidx[rowptr[i]:rowptr[i + 1]]:
            A[i, j] += 1.0
    d = 1.0 / np.sqrt(1.0 + np.diff(rowptr))
    return A * d[:, None] * d[None, :]


def close(got, ref, what, rel):
    got = got.cpu().double().numpy()
    assert np.linalg.norm(got - ref) <= rel * np.linalg.norm(ref), what


@pytest.mark.parametrize("N,K,F", [(301, 203, 19), (700, 602, 41), (400, 64, 128), (129, 33, 7)])
def test_step_matches_formulas(cuda_device, N, K, F):
    """fp32 sums of up to N + K terms against 64 bits, in the 2-norm: 1e-5."""
    c = inputs.layer_case(N, K, F, seed=N + F, mean_degree=5.0, hub_degree=30)
    r = np.random.default_rng(7)
    layer = NormedLayer(N, K, F, cuda_device)
    gamma, beta = 1 + 0.2 * r.standard_normal(K), 0.1 * r.standard_normal(K)
    b = 0.1 * r.standard_normal(F)
    for dst, src in ((layer.W, c["W"]), (layer.gamma, gamma), (layer.beta, beta), (layer.b, b)):
        dst.copy_(torch.from_numpy(np.asarray(src, np.float32)))
    gamma, beta, b = (t.cpu().double().numpy() for t in (layer.gamma, layer.beta, layer.b))
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    H = layer.forward(X, rowptr, colidx)
    A = dense(c["rowptr"], c["colidx"])
    y, _, rstd, xhat = R.forward(c["X"], gamma, beta, layer.eps)
    Wb = np.where(c["W"] >= 0, 1.0, -1.0) * np.abs(c["W"].astype(np.float64)).mean(0)
    close(H, A @ (y @ Wb + b), "H", 1e-5)
    dH = r.standard_normal((N, F)).astype(np.float32)
    dWb, db, dgamma, dbeta, dX = layer.backward(to_dev(dH), rowptr, colidx)
    v = B.checkpoint_unpack(layer.q, layer.exps).cpu().double().numpy()
    assert np.abs(v - xhat).max() <= np.abs(xhat).max() / 127.5 * 1.01
    G = A @ dH
    rw, rb = R.weight_grad(v, gamma, beta, G)
    close(dWb, rw, "dWb", 1e-5)
    close(db, rb, "db", 1e-5)
    rdx, rg, rbeta = R.backward(G @ Wb.T, gamma, v, rstd)
    close(dX, rdx, "dX", 1e-5)
    close(dgamma, rg, "dgamma", 1e-5)
    close(dbeta, rbeta, "dbeta", 1e-5)
    sign = np.where(c["W"] >= 0, 1.0, -1.0)
    scale = np.abs(c["W"].astype(np.float64)).mean(0)
    close(layer.weight_gradient(),
          sign * (rw * sign).mean(0) + scale * rw * (np.abs(c["W"]) < 1), "dW", 2e-5)


def test_gradients_follow_the_loss(cuda_device):
    """Directional differences of the 64-bit loss. The checkpoint's steps (at most 1/127.5 of a
    group's largest magnitude) are the gradients' own error: within 2 % along their directions."""
    N, K, F = 200, 96, 16
    c = inputs.layer_case(N, K, F, seed=3, mean_degree=4.0)
    layer = NormedLayer(N, K, F, cuda_device)
    layer.W.copy_(torch.from_numpy(c["W"]))
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    A = dense(c["rowptr"], c["colidx"])
    Wb = np.where(c["W"] >= 0, 1.0, -1.0) * np.abs(c["W"].astype(np.float64)).mean(0)
    target = np.random.default_rng(1).standard_normal((N, F))

    def loss(x, g, Wb):
        return 0.5 * ((A @ (R.forward(x, g, np.zeros(K), layer.eps)[0] @ Wb) - target) ** 2).sum()

    H = layer.forward(X, rowptr, colidx)
    dWb, _, dgamma, _, dX = layer.backward(H - to_dev(target.astype(np.float32)), rowptr, colidx)
    x, g = c["X"].astype(np.float64), np.ones(K)
    h = 1e-5
    for grad, at in ((dX, lambda d: loss(x + d, g, Wb)), (dgamma, lambda d: loss(x, g + d, Wb)),
                     (dWb, lambda d: loss(x, g, Wb + d))):
        d = grad.cpu().double().numpy()
        d /= np.linalg.norm(d)
        slope = (at(h * d) - at(-h * d)) / (2 * h)
        assert abs(slope - np.linalg.norm(grad.cpu().double().numpy())) <= 0.02 * abs(slope)


def test_capture_replays(cuda_device):
    """The whole step in a CUDA graph: no call allocates or synchronises."""
    N, K, F = 500, 130, 24
    c = inputs.layer_case(N, K, F, seed=5, mean_degree=4.0)
    layer = NormedLayer(N, K, F, cuda_device)
    layer.W.copy_(torch.from_numpy(c["W"]))
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    dH = torch.ones((N, F), device=cuda_device)

    def step():
        layer.forward(X, rowptr, colidx)
        layer.backward(dH, rowptr, colidx)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    want = [t.clone() for t in (layer.dWb, layer.dX, layer.dgamma)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (layer.dWb, layer.dX, layer.dgamma):
        t.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (layer.dWb, layer.dX, layer.dgamma)))
