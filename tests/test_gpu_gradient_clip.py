"""runner.GradientClip over layers of both kinds: the norm is that of the gradients that a step applies to the
parameters, a normed layer's W among them, whose gradient goes through the sign."""
import numpy as np
import pytest
import torch

import residual_reference as R
from gpu_helpers import to_dev
from norm_reference import U
from paper_2010_07565_gb300 import inputs
from paper_2010_07565_gb300.runner import GradientClip, NormedLayer
from test_gpu_norm import within
from test_gpu_residual_layer import f64, made

pytestmark = pytest.mark.gpu


def layers_of_both_kinds(N, K, F, device):
    first, second = made(N, K, K, device), NormedLayer(N, K, F, device)
    # (Some magnitudes are past 1, where the sign's gradient is 0.)
    second.W.copy_(to_dev(np.random.default_rng(1).uniform(-1.2, 1.2, (K, F)).astype(np.float32)))
    return first, second


def case(N, K, device):
    c = inputs.layer_case(N, K, K, seed=9, mean_degree=4.0)
    return [to_dev(c[n]) for n in ("X", "rowptr", "colidx")]


def step(layers, X, rowptr, colidx):
    first, second = layers
    h = second.forward(first.forward(X, rowptr, colidx), rowptr, colidx)
    first.backward(second.backward(torch.tanh(h), rowptr, colidx)[-1], rowptr, colidx)


def weight_gradient(layer):
    """dL/dW in 64 bits from the layer's dWb, and the error of fp32: a mean of K terms in any order, the
    column's scale of K terms, and five operations."""
    W, d, K = f64(layer.W), f64(layer.dWb), layer.K
    sign = np.where(W >= 0, 1.0, -1.0)
    through = np.abs(W).mean(0) * d * (np.abs(W) < 1)
    return sign * (d * sign).mean(0) + through, \
        (K + 5) * U * (np.abs(d).mean(0) + np.abs(through))


@pytest.mark.parametrize("limit", [2.0 ** -10, 2.0 ** 20])
def test_limits_the_parameters_gradients(cuda_device, limit):
    """The factor is off from that of the rounded norm by three roundings (norm, factor, product)."""
    N, K, F = 300, 64, 8
    layers = layers_of_both_kinds(N, K, F, cuda_device)
    clip = GradientClip(layers)
    X, rowptr, colidx = case(N, K, cuda_device)
    first, second = layers
    for _ in range(2):                      # (the second: gradients that were scaled are written anew)
        step(layers, X, rowptr, colidx)
        dW, error = weight_gradient(second)
        dWb = second.dWb.clone()
        want = [f64(g) for g in (first.dW, first.db, first.dgamma)] + [dW] + \
            [f64(g) for g in (second.db, second.dgamma, second.dbeta)]
        norm = np.sqrt(sum((w ** 2).sum() for w in want))
        got = clip(limit).item()
        slack = np.sqrt((error ** 2).sum()) + R.NORM_ERROR * norm
        assert abs(got - norm) <= slack
        factor = min(1.0, limit / got)
        grads = first.gradients() + second.gradients()
        for g, w in zip(grads, want):
            e = 3.01 * U * np.abs(w * factor) + (error * factor if w is dW else 0.0)
            within(g, w * factor, e, "gradient")
        assert (factor == 1.0) == (limit > 1)
        total = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
        assert factor == 1.0 or abs(total - limit) <= (R.NORM_ERROR + 4 * U) * limit
        assert torch.equal(second.dWb, dWb)
        assert [g.shape for g in second.gradients()] == \
            [p.shape for p in (second.W, second.b, second.gamma, second.beta)]


def test_captured_with_the_step(cuda_device):
    N, K, F = 300, 64, 8
    layers = layers_of_both_kinds(N, K, F, cuda_device)
    clip = GradientClip(layers)
    X, rowptr, colidx = case(N, K, cuda_device)

    def run():
        step(layers, X, rowptr, colidx)
        clip(2.0 ** -10)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    tensors = [clip.norm] + layers[0].gradients() + layers[1].gradients()
    want = [t.clone() for t in tensors]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(2):
        for t in tensors:
            t.fill_(float("nan"))
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, tensors))


def test_weight_gradient_behind_the_clipping_is_clipped(cuda_device):
    """A step that asks weight_gradient() again gets what the list holds, in a tensor of its own; a layer whose
    gradients nobody asked for has dWb's."""
    N, K, F = 300, 64, 8
    layers = layers_of_both_kinds(N, K, F, cuda_device)
    X, rowptr, colidx = case(N, K, cuda_device)
    second = layers[1]
    step(layers, X, rowptr, colidx)
    whole = second.weight_gradient()
    within(whole, *weight_gradient(second), "gradient of W")
    clip = GradientClip(layers)
    for limit in (2.0 ** -10, 2.0 ** -12):
        norm = clip(limit).item()
        got = second.weight_gradient()
        assert torch.equal(got, second.dW) and norm > limit
        assert got.abs().max() < 0.5 * whole.abs().max()
        got.zero_()
        assert second.dW.abs().max() > 0
        step(layers, X, rowptr, colidx)
        assert torch.equal(second.weight_gradient(), whole)


def test_weight_gradient_is_kept_for_those_who_ask(cuda_device):
    """Asked for after a backward pass, gradients() has that pass's and from then on every later one's; a
    graph that was captured before cannot write it, which is refused."""
    N, K, F = 300, 64, 8
    layers = layers_of_both_kinds(N, K, F, cuda_device)
    X, rowptr, colidx = case(N, K, cuda_device)
    second = layers[1]
    for scale in (1.0, 3.0):
        step(layers, scale * X, rowptr, colidx)
        want = second.weight_gradient()
        kept = second.gradients()[0]
        assert torch.equal(kept, want) and kept.data_ptr() == second.gradients()[0].data_ptr()
    layers = layers_of_both_kinds(N, K, F, cuda_device)
    step(layers, X, rowptr, colidx)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(layers, X, rowptr, colidx)
    g.replay()
    with pytest.raises(RuntimeError, match="before capturing"):
        GradientClip(layers)
    torch.cuda.synchronize()
