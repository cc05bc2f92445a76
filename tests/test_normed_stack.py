"""Layers of a stack in training that share their scratch (runner.NormedScratch): what they keep is
the 8-bit checkpoints, and the gradients are those of layers with memory of their own."""
import numpy as np
import pytest
import torch

from paper_2010_07565_gb300 import binding as B
from paper_2010_07565_gb300 import build as lib_build
from paper_2010_07565_gb300 import inputs
from paper_2010_07565_gb300.runner import NormedLayer, NormedScratch

SIZES = [(203, 96), (96, 96), (96, 19)]          # K, F of a stack's layers


def stack(N, device, shared):
    sizes = [(N, K, F) for K, F in SIZES]
    scratch = NormedScratch(sizes, device) if shared else None
    return [NormedLayer(*size, device, scratch=scratch) for size in sizes]


def bytes_of(layers):
    """Bytes of the distinct buffers that the layers hold."""
    seen = {}
    for layer in layers:
        for t in vars(layer).values():
            if isinstance(t, torch.Tensor):
                store = t.untyped_storage()
                seen[store.data_ptr()] = store.nbytes()
    return sum(seen.values())


def test_a_stack_keeps_checkpoints_not_rows():
    """Beyond what does not grow with N: a layer's checkpoint (33/32 bytes a value, rows padded),
    rstd and H, and the scratch once."""
    lib_build.build()
    small, big = 1 << 12, 1 << 14
    grown = bytes_of(stack(big, "cpu", True)) - bytes_of(stack(small, "cpu", True))
    pad = lambda n, m: -(-n // m) * m
    kept = sum(pad(K, 16) + pad(-(-K // 32), 4) + 4 + 4 * F for K, F in SIZES)
    scratch = 4 * max(2 * K for K, _ in SIZES) + 4 * max(F for _, F in SIZES)
    work = [max(max(B.bigcn_layer_norm_backward_workspace_bytes(N, K),
                    B.bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F)) for K, F in SIZES)
            for N in (small, big)]
    assert grown == (big - small) * (kept + scratch) + work[1] - work[0]
    own = bytes_of(stack(big, "cpu", False)) - bytes_of(stack(small, "cpu", False))
    assert grown < own


@pytest.mark.gpu
def test_shared_scratch_gives_the_same_gradients(cuda_device):
    N = 400
    c = inputs.layer_case(N, 203, 96, seed=4, mean_degree=5.0, hub_degree=30)
    t = lambda a: torch.from_numpy(np.asarray(a)).to(cuda_device)
    X, rowptr, colidx = t(c["X"]), t(c["rowptr"]), t(c["colidx"])
    r = np.random.default_rng(2)
    weights = [r.uniform(-1, 1, size).astype(np.float32) for size in SIZES]
    dH = t(r.standard_normal((N, SIZES[-1][1])).astype(np.float32))
    results = []
    for shared in (False, True):
        layers, h, out = stack(N, cuda_device, shared), X, []
        for layer, w in zip(layers, weights):
            layer.W.copy_(t(w))
            h = layer.forward(h, rowptr, colidx)
        out.append(h.clone())
        d = dH
        for layer in reversed(layers):
            grads = layer.backward(d, rowptr, colidx)
            out += [g.clone() for g in grads]
            d = grads[-1]
        results.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert all(torch.isfinite(a).all() for a in results[0])
