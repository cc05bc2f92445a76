"""The norm of many tensors together and their scaling, on the GPU against 64 bits within the bounds that
residual_reference derives."""
import numpy as np
import pytest
import torch

import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, f64, within

pytestmark = pytest.mark.gpu

NAMES = {v: k for k, v in DTYPES.items()}


def tensors(shapes, seed, device, scale=1.0):
    """shapes: (type, shape) pairs."""
    r = np.random.default_rng(seed)
    return [torch.from_numpy((scale * r.standard_normal(s)).astype(np.float32)).to(DTYPES[d]).to(device)
            for d, s in shapes]


LISTS = {
    "one": [("float32", (1,))],
    "two layers": [("float32", (1433, 64)), ("float32", (64,)), ("float32", (64, 7)), ("float32", (7,))],
    "mixed": [("bfloat16", (602, 128)), ("float32", (128,)), ("float16", (33, 5)), ("float32", (0,)),
              ("bfloat16", (1,)), ("float32", (4096 * 4,)), ("float16", (8191,))],
    "large": [("float32", (3000, 1001)), ("bfloat16", (4001, 999)), ("float16", (2, 1 << 20))],
    "many": [("float32" if i % 3 else "bfloat16", (1 + 37 * i % 501,)) for i in range(2100)],
}


def check(ts, norm, outs, max_norm):
    want, ref = R.clip([f64(t) for t in ts], max_norm)
    within(norm, np.array([want]), np.array([want * R.NORM_ERROR]), "norm")
    for i, (o, w, t) in enumerate(zip(outs, ref, ts)):
        if want <= max_norm:
            assert torch.equal(o, t)
        else:
            within(o, w, R.clip_bound(w, NAMES[t.dtype]), f"tensor {i}")


@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e30])
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clip(cuda_device, name, max_norm):
    ts = tensors(LISTS[name], 3, cuda_device)
    first = B.grad_norm(ts)
    outs = [torch.full_like(t, 7.0) for t in ts]
    ws = torch.full((B.bigcn_grad_norm_workspace_bytes(ts) // 8,), float("nan"), dtype=torch.float64,
                    device=cuda_device)
    norm = torch.empty(1, device=cuda_device)
    kept = [t.clone() for t in ts]
    B.bigcn_clip_grad_norm(ts, max_norm, norm, ws, out=outs)
    assert torch.equal(norm, first) and all(torch.equal(a, b) for a, b in zip(ts, kept))
    check(ts, norm, outs, max_norm)
    again = B.clip_grad_norm(ts, max_norm)               # in place
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(ts, outs))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offset,out_offset", [(0, 0), (1, 1), (3, 0), (0, 5), (7, 2)])
def test_offsets(cuda_device, offset, out_offset, dtype):
    """Tensors that start anywhere; what lies around them is not written."""
    r = np.random.default_rng(offset)
    ins, outs, bufs = [], [], []
    for n in (1, 2, 15, 100, 4096, 4097, 20001, 65536 + 3):
        v = torch.from_numpy(r.standard_normal(n).astype(np.float32)).to(DTYPES[dtype])
        a = torch.full((n + 32,), float("nan"), dtype=DTYPES[dtype], device=cuda_device)
        b = torch.full((n + 32,), 7.0, dtype=DTYPES[dtype], device=cuda_device)
        a[offset:offset + n] = v.to(cuda_device)
        ins.append(a[offset:offset + n])
        outs.append(b[out_offset:out_offset + n])
        bufs.append(b)
    norm, ws = torch.empty(1, device=cuda_device), torch.empty(8192, dtype=torch.uint8, device=cuda_device)
    B.bigcn_clip_grad_norm(ins, 2.0, norm, ws, out=outs)
    check(ins, norm, outs, 2.0)
    for o, b in zip(outs, bufs):
        o.fill_(7.0)
        assert (b == 7.0).all()


@pytest.mark.parametrize("dtype,scale", [("float32", 1e-40), ("float32", 1e-30), ("float32", 1e-19),
                                         ("float32", 1e25), ("float32", 1e35), ("bfloat16", 1e-38),
                                         ("bfloat16", 1e34), ("float16", 1e-6)])
def test_ranges(cuda_device, dtype, scale):
    """Elements whose squares leave fp32, alone and beside ordinary ones."""
    big = tensors([(dtype, (70001,)), (dtype, (33,))], 1, cuda_device, scale)
    check(big, B.grad_norm(big), [], 1.0)
    # (At 1e-40 the gradients are subnormal, and their norm is one too: an absolute step of 2^-149.)
    mixed = big + tensors([("float32", (500,))], 2, cuda_device)
    want = R.clip([f64(t) for t in mixed], 1.0)[0]
    within(B.grad_norm(mixed), np.array([want]), np.array([want * R.NORM_ERROR]), "norm")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_not_finite(cuda_device, bad):
    """A NaN or an infinity anywhere: the norm says so and the tensors stay as they are."""
    ts = tensors(LISTS["mixed"], 5, cuda_device)
    ts[4][0] = bad
    kept = [t.clone() for t in ts]
    norm = B.clip_grad_norm(ts, 0.1)
    assert torch.isnan(norm).all() if bad != bad else torch.isinf(norm).all()
    outs = [torch.zeros_like(t) for t in ts]
    ws = torch.empty(B.bigcn_grad_norm_workspace_bytes(ts), dtype=torch.uint8, device=cuda_device)
    B.bigcn_clip_grad_norm(ts, 0.1, norm, ws, out=outs)
    for a, b, c in zip(ts, kept, outs):
        bits = torch.int32 if a.dtype == torch.float32 else torch.int16
        assert torch.equal(a.view(bits), b.view(bits)) and torch.equal(c.view(bits), b.view(bits))


def test_nothing_to_add(cuda_device):
    for ts in ([], [torch.empty(0, device=cuda_device)], [torch.zeros(1000, device=cuda_device)]):
        assert B.grad_norm(ts).item() == 0.0 and B.clip_grad_norm(ts, 1.0).item() == 0.0


def test_norm_counts_a_tensor_as_often_as_listed(cuda_device):
    t = tensors([("float32", (1000,))], 8, cuda_device)[0]
    a, b = B.grad_norm([t]).item(), B.grad_norm([t, t[500:], t[:500]]).item()
    assert abs(b - a * 2 ** 0.5) <= 4e-7 * b


def test_repeats_capture_and_streams(cuda_device):
    """The same bits in every call; a captured call holds its list and works on new values; two calls at
    once with workspaces of their own."""
    ts = tensors(LISTS["large"], 4, cuda_device)
    kept = [t.clone() for t in ts]
    lists = B.TensorList(ts)
    new = lambda: (torch.empty(1, device=cuda_device),
                   torch.empty(B.bigcn_grad_norm_workspace_bytes(lists), dtype=torch.uint8,
                               device=cuda_device))
    norm, ws = new()
    B.bigcn_clip_grad_norm(lists, 1.0, norm, ws)
    want = norm.item(), [t.clone() for t in ts]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.bigcn_clip_grad_norm(lists, 1.0, norm, ws)
    del lists
    for _ in range(3):
        for t, k in zip(ts, kept):
            t.copy_(k)
        g.replay()
        torch.cuda.synchronize()
        assert norm.item() == want[0] and all(torch.equal(a, b) for a, b in zip(ts, want[1]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    lists = [B.TensorList(kept), B.TensorList(kept[:1])]
    bufs = [
        (torch.empty(1, device=cuda_device), torch.empty(1 << 16, dtype=torch.uint8, device=cuda_device))
        for _ in range(2)]
    alone = [B.grad_norm(l).item() for l in lists]
    torch.cuda.synchronize()
    for _ in range(20):
        for l, (n, w), s in zip(lists, bufs, streams):
            B.bigcn_grad_norm(l, n, w, stream=s)
    torch.cuda.synchronize()
    assert [n.item() for n, _ in bufs] == alone
