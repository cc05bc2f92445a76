"""Residual layers in training (runner.ResidualLayer): the stream's addition and RMS norm, the product in
4 bits, the aggregation, every gradient and their clipping, as a stack uses them, against 64-bit
formulas over a dense adjacency and the same 4-bit operands and checkpoints."""
import numpy as np
import pytest
import torch

import norm_reference as N_
import residual_reference as R
from gpu_helpers import to_dev
from paper_2010_07565_gb300 import binding as B
from paper_2010_07565_gb300 import inputs
from paper_2010_07565_gb300.runner import GradientClip, NormedLayer, ResidualLayer, ResidualScratch
from test_gpu_normed_layer import close, dense

pytestmark = pytest.mark.gpu


def f64(t):
    return t.cpu().double().numpy()


def made(N, K, F, device, seed=7):
    r = np.random.default_rng(seed)
    layer = ResidualLayer(N, K, F, device)
    for dst, src in ((layer.W, r.uniform(-1, 1, (K, F)) / np.sqrt(K)), (layer.b, 0.1 * r.standard_normal(F)),
                     (layer.gamma, 1 + 0.2 * r.standard_normal(K))):
        dst.copy_(torch.from_numpy(src.astype(np.float32)))
    return layer


def values4(kept, K):
    return R.fp4_values(R.fp4_codes(kept[0].cpu().numpy(), K), kept[1].cpu().numpy())


@pytest.mark.parametrize("N,K,F", [(301, 203, 19), (700, 602, 41), (400, 64, 128), (129, 33, 7)])
def test_step_matches_formulas(cuda_device, N, K, F):
    """fp32 sums of up to N + K terms against 64 bits, in the 2-norm: 1e-5."""
    c = inputs.layer_case(N, K, F, seed=N + F, mean_degree=5.0, hub_degree=30)
    r = np.random.default_rng(3)
    layer = made(N, K, F, cuda_device)
    gamma, b = f64(layer.gamma), f64(layer.b)
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    stream = to_dev(r.standard_normal((N, K)).astype(np.float32))
    s = f64(X + stream)
    H = layer.forward(X, rowptr, colidx, R=stream)
    A = dense(c["rowptr"], c["colidx"])
    assert np.array_equal(f64(stream), s)
    y, rstd, shat = R.rms_forward(s, gamma, layer.eps)
    close(layer.Y, y, "Y", 1e-6)
    y4, w4 = values4(layer.y4, K), values4(layer.w4, K)
    assert np.array_equal(y4, R.fp4_values(*R.fp4_pack(f64(layer.Y))))
    assert np.array_equal(w4, R.fp4_values(*R.fp4_pack(f64(layer.W).T)))
    close(H, A @ (y4 @ w4.T + b), "H", 1e-5)
    dH, dS = (r.standard_normal((N, w)).astype(np.float32) for w in (F, K))
    past = to_dev(dS)
    dW, db, dgamma, dX = layer.backward(to_dev(dH), rowptr, colidx, dS=past)
    assert dX.data_ptr() == past.data_ptr()
    v = f64(B.checkpoint_unpack(layer.q, layer.exps))
    assert np.abs(v - shat).max() <= np.abs(shat).max() / 127.5 * 1.01
    G = A @ dH
    close(layer.G, G, "G", 1e-5)
    rw, rb = N_.weight_grad(v, gamma, np.zeros(K), G)
    close(dW, rw, "dW", 1e-5)
    close(db, rb, "db", 1e-5)
    g4, wr = values4(layer.g4, F), values4(layer.w4_rows, F)
    assert np.array_equal(wr, R.fp4_values(*R.fp4_pack(f64(layer.W))))
    dy = g4 @ wr.T
    rdx, rg = R.rms_backward(dy, gamma, v, rstd, dS)
    close(dX, rdx, "dX", 1e-5)
    close(dgamma, rg, "dgamma", 1e-5)


def stack_step(layers, clip, X, dH, rowptr, colidx):
    """Forward and backward of a stack whose layers but the last have as many outputs as inputs."""
    stream, h = X.clone(), layers[0].forward(X, rowptr, colidx)
    for layer in layers[1:]:
        h = layer.forward(h, rowptr, colidx, R=stream)
    d, past = dH, None
    for layer in reversed(layers):
        d = layer.backward(d, rowptr, colidx, dS=past)[-1]
        past = d
    return h, d, clip(0.3)


def stack(N, sizes, device, shared):
    scratch = ResidualScratch([(N, K, F) for K, F in sizes], device) if shared else None
    layers = []
    for i, (K, F) in enumerate(sizes):
        layer = made(N, K, F, device, seed=i)
        if shared:
            kept = {n: getattr(layer, n).clone() for n in ("W", "b", "gamma")}
            layer = ResidualLayer(N, K, F, device, scratch=scratch)
            for n, t in kept.items():
                getattr(layer, n).copy_(t)
        layers.append(layer)
    return layers


def test_a_stack_with_shared_scratch_and_in_a_graph(cuda_device):
    """A stack's step, its gradients clipped together: with scratch of each layer's own, shared, and
    captured and replayed, the same bits; the clipped gradients' norm is the limit."""
    N, sizes = 400, [(96, 96), (96, 96), (96, 19)]
    c = inputs.layer_case(N, 96, 96, seed=4, mean_degree=5.0, hub_degree=30)
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    dH = to_dev(np.random.default_rng(2).standard_normal((N, 19)).astype(np.float32))
    results = []
    for shared in (False, True):
        layers = stack(N, sizes, cuda_device, shared)
        clip = GradientClip(layers)
        h, d, norm = stack_step(layers, clip, X, dH, rowptr, colidx)
        results.append([t.clone() for t in (h, d, norm, *clip.list.tensors)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert all(torch.isfinite(t).all() for t in results[0])
    assert results[0][2].item() > 0.3
    total = np.sqrt(sum((f64(t) ** 2).sum() for t in clip.list.tensors))
    assert abs(total - 0.3) <= 0.3 * 1e-6
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        stack_step(layers, clip, X, dH, rowptr, colidx)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h, d, norm = stack_step(layers, clip, X, dH, rowptr, colidx)
    for t in (h, d, norm, *clip.list.tensors):
        t.fill_(float("nan"))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results[1], (h, d, norm, *clip.list.tensors)))
    assert B.device_timeouts() == 0


def test_descent_with_clipped_steps_runs(cuda_device):
    """Steps against the gradients, clipped, with layers of both kinds in one list: everything stays
    finite."""
    N, K = 300, 64
    c = inputs.layer_case(N, K, K, seed=9, mean_degree=4.0)
    X, rowptr, colidx = to_dev(c["X"]), to_dev(c["rowptr"]), to_dev(c["colidx"])
    first, second = made(N, K, K, cuda_device), NormedLayer(N, K, 8, cuda_device)
    second.W.copy_(to_dev(np.random.default_rng(1).uniform(-1, 1, (K, 8)).astype(np.float32)))
    clip = GradientClip([first, second])
    for _ in range(4):
        h = second.forward(first.forward(X, rowptr, colidx), rowptr, colidx)
        first.backward(second.backward(torch.tanh(h), rowptr, colidx)[-1], rowptr, colidx)
        norm = clip(1.0)
        for layer in (first, second):
            for p, g in zip((layer.W, layer.b, layer.gamma), layer.gradients()):
                p -= 0.1 * g
        assert torch.isfinite(norm).all() and all(torch.isfinite(t).all() for t in clip.list.tensors)
