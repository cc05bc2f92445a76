"""Two-layer Bi-GCN forward on one GPU: device buffers, the C-ABI calls and
their CUDA-graph capture.

Plumbing around libbigcn.so: torch owns the device memory and the stream,
and every step of the computation runs in the library's kernels.

``launch()`` makes the one call ``bigcn_forward_2layer`` (4 kernels for the
usual widths: both weight packs; layer-1 centre + pack + XNOR GEMM; layer-1
aggregation fused with layer 2's pack and GEMM; layer-2 aggregation).
``launch_steps()`` runs the same forward as eight separate step calls
(pack_rows, pack_weights, xnor_gemm_degscaled, spmm_prescaled per layer),
keeping every intermediate in its own buffer, for step-by-step checks.
The output is the logits (no softmax: Eq. 2 belongs to training).

:class:`NormedLayer` is one layer in training whose features stay real (only the weights
binarized) and whose input rows are normalised: layer norm, product, aggregation and their
gradients, with the normalised rows kept in 8 bits in between.

:class:`ResidualLayer` is one layer of a deep residual stack in training: it adds its input to the
stream of rows that all layers share, normalises the sum, multiplies in 4 bits and aggregates;
:class:`GradientClip` scales the gradients of such a stack by their common norm.
"""
from __future__ import annotations

import torch

from . import binding as B

STEP_KERNELS = ("pack_rows", "pack_weights", "xnor_gemm", "spmm")


FRONT = "L1.pack_rows+L1.xnor_gemm"
FUSED_AGG = "L1.spmm+L2.pack_rows+L2.xnor_gemm"


def fused_kernel_names(N: int, K: int, Fh: int, Fo: int):
    """Names of the kernels bigcn_forward_2layer launches for these sizes, in
    order (4 to 7 of them, depending on which fusions the widths allow)."""
    n = B.bigcn_forward_2layer_launches(N, K, Fh, Fo)
    front_fused = n in (4, 6)
    agg_fused = n in (4, 5)
    names = ["pack_weights(W1,W2)"]
    names += [FRONT] if front_fused else ["L1.pack_rows", "L1.xnor_gemm"]
    names += [FUSED_AGG] if agg_fused else ["L1.spmm", "L2.pack_rows", "L2.xnor_gemm"]
    names += ["L2.spmm"]
    return tuple(names)


class GCN2Forward:
    """Buffers and launch sequence of the 2-layer Bi-GCN forward of Sec. 6.2."""

    def __init__(self, N: int, K: int, hidden: int, out: int, nnz: int, device,
                 keep_h1: bool = False):
        self.N, self.K, self.hidden, self.out, self.nnz = N, K, hidden, out, nnz
        self.device = torch.device(device)
        f32, i64 = torch.float32, torch.int64
        e = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=self.device)
        # inputs
        self.X, self.s, self.t = e(N, K), e(K), e(K)
        self.W1, self.W2 = e(K, hidden), e(hidden, out)
        self.rowptr, self.colidx = e(N + 1, dtype=i64), e(max(nnz, 1), dtype=torch.int32)[:nnz]
        # fused forward
        nbytes = B.bigcn_forward_2layer_workspace_bytes(N, K, hidden, out)
        self.workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=self.device)
        self.logits = e(N, out)
        self.H1 = e(N, hidden) if keep_h1 else None
        self.kernel_names = fused_kernel_names(N, K, hidden, out)
        self.graph = None
        self._steps = None

    def input_tensors(self):
        return dict(X=self.X, s=self.s, t=self.t, W1=self.W1, W2=self.W2,
                    rowptr=self.rowptr, colidx=self.colidx)

    def load(self, non_blocking: bool = True, **tensors):
        """Copy inputs (host, pinned host or device tensors) into the buffers."""
        dst = self.input_tensors()
        for name, src in tensors.items():
            dst[name].copy_(src, non_blocking=non_blocking)

    def launch(self, events=None):
        """Enqueue the fused forward on the current stream; ``events`` (len =
        launches + 1) are recorded before each kernel and after the last."""
        B.bigcn_forward_2layer(self.X, self.s, self.t, self.W1, self.W2, self.rowptr,
                               self.colidx, self.workspace, self.logits, H1=self.H1,
                               events=events)

    def capture(self, events=None):
        """Capture launch(events) into a CUDA graph (replayed by replay())."""
        if events:
            for ev in events:       # torch creates the CUDA event on first record
                ev.record()
        s = torch.cuda.Stream(device=self.device)
        s.wait_stream(torch.cuda.current_stream(self.device))
        with torch.cuda.stream(s):
            self.launch(events)     # warm-up outside the graph
        torch.cuda.current_stream(self.device).wait_stream(s)
        torch.cuda.synchronize(self.device)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.launch(events)
        self.graph = g
        return g

    def replay(self):
        self.graph.replay()

    # ----------------------------------------------------- step by step ----
    def _alloc_steps(self):
        N, K, Fh, Fo = self.N, self.K, self.hidden, self.out
        f32, i64 = torch.float32, torch.int64
        e = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=self.device)
        w1, w2 = B.words_for(K), B.words_for(Fh)
        self._steps = True
        self.bits1, self.alpha1 = e(N, w1, dtype=i64), e(N)
        self.wbits1, self.beta1 = e(Fh, w1, dtype=i64), e(Fh)
        self.Z1, self.H1s = e(N, Fh), e(N, Fh)
        self.bits2, self.alpha2 = e(N, w2, dtype=i64), e(N)
        self.wbits2, self.beta2 = e(Fo, w2, dtype=i64), e(Fo)
        self.Z2, self.logits_steps = e(N, Fo), e(N, Fo)

    def launch_steps(self):
        """The same forward as eight step calls, every intermediate kept."""
        if self._steps is None:
            self._alloc_steps()
        B.bigcn_pack_rows(self.X, self.s, self.t, self.bits1, self.alpha1)
        B.bigcn_pack_weights(self.W1, self.wbits1, self.beta1)
        B.bigcn_xnor_gemm_degscaled(self.bits1, self.alpha1, self.wbits1, self.beta1, self.K,
                                    self.rowptr, self.Z1)
        B.bigcn_spmm_prescaled(self.rowptr, self.colidx, self.Z1, self.H1s)
        B.bigcn_pack_rows(self.H1s, None, None, self.bits2, self.alpha2)
        B.bigcn_pack_weights(self.W2, self.wbits2, self.beta2)
        B.bigcn_xnor_gemm_degscaled(self.bits2, self.alpha2, self.wbits2, self.beta2,
                                    self.hidden, self.rowptr, self.Z2)
        B.bigcn_spmm_prescaled(self.rowptr, self.colidx, self.Z2, self.logits_steps)


class NormedScratch:
    """What layers of a stack need only within a call: the largest layer's Y (and dY), Z (and
    G), dX and workspace, for ``sizes``, the layers' (N, K, F). Layers that are given one share
    it, on one stream; dX holds a layer's gradient until the layer below has run its backward."""

    def __init__(self, sizes, device):
        sizes = list(sizes)
        e = lambda n, dtype=torch.float32: torch.empty(n, dtype=dtype, device=torch.device(device))
        most = lambda f: max(f(*size) for size in sizes)
        self.Y, self.dX = (e(most(lambda N, K, F: N * K)) for _ in range(2))
        self.Z = e(most(lambda N, K, F: N * F))
        self.workspace = e(most(lambda N, K, F: max(
            B.bigcn_layer_norm_backward_workspace_bytes(N, K),
            B.bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F), 1)), dtype=torch.uint8)


class NormedLayer:
    """One layer in training, H = A~ (Y W~ + b) with Y = gamma xhat + beta the layer norm of X
    and W~ = diag(beta_j) sign(W) (the ablation that binarizes the weights only, Sec. 6.3).

    Between ``forward()`` and ``backward()`` it keeps xhat's 8-bit checkpoint and each row's
    rstd: N (K + K/32 + 4) bytes in place of the 4 N K of Y. Y, Z and dX are scratch, of the
    layer's own or, for the layers of a stack, of one ``scratch`` (a :class:`NormedScratch`)
    that they share. The one checkpoint serves both gradients that need the features:

        G   = A~ dH                                       (the CSR is symmetric)
        dWb = dL/dW~ = Y^T G,   db = sum_i G_i            (Algorithm 1's dL/dW~ with real features)
        dY  = G W~^T
        dX, dgamma, dbeta                                 the norm's gradients from dY

    ``weight_gradient()`` is dWb taken through the sign (Eq. bp-W): the gradient of W itself, which a step
    subtracts. Once ``gradients()`` has been asked for, ``backward()`` writes it into dW each time."""

    def __init__(self, N: int, K: int, F: int, device, eps: float = 1e-5, scratch=None):
        self.N, self.K, self.F, self.eps = N, K, F, eps
        self.device = torch.device(device)
        f32, i64 = torch.float32, torch.int64
        e = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=self.device)
        # parameters
        self.W, self.b = e(K, F), torch.zeros(F, device=self.device)
        self.gamma, self.beta = torch.ones(K, device=self.device), torch.zeros(K, device=self.device)
        # kept from forward to backward
        self.q, self.exps = B.checkpoint_buffers(N, K, self.device)
        self.rstd = e(N)
        self.w_bits, self.w_scale = e(F, B.words_for(K), dtype=i64), e(F)
        self.H = e(N, F)
        # scratch: free for other layers between calls (dX until the layer below has read it)
        scratch = scratch or NormedScratch([(N, K, F)], self.device)
        take = lambda t, cols: t[:N * cols].view(N, cols)
        self.Y, self.Z, self.dX = take(scratch.Y, K), take(scratch.Z, F), take(scratch.dX, K)
        self.workspace = scratch.workspace
        # gradients
        self.G, self.dY = self.Z, self.Y
        self.dWb, self.db = e(K, F), e(F)
        self.dgamma, self.dbeta = e(K), e(K)
        self.dW, self._captured = None, False
        self.w_rows, self.w_rows_scale = e(K, B.words_for(F), dtype=i64), e(K)
        self.one, self.zero = torch.ones(K, device=self.device), torch.zeros(F, device=self.device)

    def forward(self, X, rowptr, colidx):
        """H from X (N x K fp32); enqueued on the current stream."""
        B.bigcn_layer_norm_forward(X, self.gamma, self.beta, self.eps, self.Y, rstd=self.rstd,
                                   q=self.q, exps=self.exps)
        B.bigcn_pack_weights(self.W, self.w_bits, self.w_scale)
        B.bigcn_real_binary_gemm(self.Y, None, None, self.w_bits, self.w_scale, self.Z)
        self.Z += self.b
        B.bigcn_spmm_norm(rowptr, colidx, self.Z, self.H)
        return self.H

    def backward(self, dH, rowptr, colidx):
        """The gradients (dWb, db, dgamma, dbeta, dX) from dH = dL/dH (N x F)."""
        B.bigcn_spmm_norm(rowptr, colidx, dH, self.G)
        B.bigcn_checkpoint_weight_grad(self.q, self.exps, self.G, self.workspace, self.dWb,
                                       gamma=self.gamma, beta=self.beta, db=self.db)
        # (Ten torch calls, 110 us of the host's time beside 60 for the rest: for those who ask.)
        if self.dW is not None:
            self._through_sign(self.dW)
        elif torch.cuda.is_current_stream_capturing():
            self._captured = True
        # dY = (G diag(beta_j)) sign(W)^T: W packed row by row over its F columns.
        B.bigcn_pack_rows(self.W, None, None, self.w_rows, self.w_rows_scale)
        B.bigcn_real_binary_gemm(self.G, self.w_scale, self.zero, self.w_rows, self.one, self.dY)
        B.bigcn_layer_norm_backward(self.dY, self.gamma, self.rstd, self.workspace, q=self.q,
                                    exps=self.exps, dX=self.dX, dgamma=self.dgamma,
                                    dbeta=self.dbeta)
        return self.dWb, self.db, self.dgamma, self.dbeta, self.dX

    def gradients(self):
        """The parameters' gradients, in the order W, b, gamma, beta: buffers that ``backward()`` writes
        from the first call on. A captured ``backward()`` does so only if they had been asked for."""
        if self.dW is None:
            if self._captured:
                raise RuntimeError("a captured backward() leaves dW out: ask for gradients() before capturing")
            self.dW = self._through_sign()
        return [self.dW, self.db, self.dgamma, self.dbeta]

    def weight_gradient(self):
        """The gradient of W, a tensor of its own: of dW where ``gradients()`` has been asked for, scaled as that
        has been since (``GradientClip``), else of dWb as it is."""
        return self._through_sign() if self.dW is None else self.dW.clone()

    def _through_sign(self, out=None):
        """Eq. bp-W of dWb: sign(W) times the column means of dWb sign(W), and beta_j dWb where
        |W| < 1 (the straight-through estimator of sign)."""
        sign = torch.where(self.W >= 0, 1.0, -1.0)
        return torch.add(sign * (self.dWb * sign).mean(0),
                         self.w_scale * self.dWb * (self.W.abs() < 1), out=out)


class ResidualScratch:
    """What layers of a residual stack need only within a call: the largest layer's Y (and dY), Z
    (and G), the 4-bit rows of Y, G and the weights, and workspace, for ``sizes``, the layers' (N, K,
    F). Layers that are given one share it, on one stream."""

    def __init__(self, sizes, device):
        sizes = list(sizes)
        e = lambda n, dtype=torch.float32: torch.empty(n, dtype=dtype, device=torch.device(device))
        most = lambda f: max(f(*size) for size in sizes)
        self.Y, self.dX = (e(most(lambda N, K, F: N * K)) for _ in range(2))
        self.Z = e(most(lambda N, K, F: N * F))
        self.rows4 = e(most(lambda N, K, F: max(_fp4_bytes(N, K), _fp4_bytes(N, F))), torch.uint8)
        self.weights4 = e(most(lambda N, K, F: max(_fp4_bytes(F, K), _fp4_bytes(K, F))), torch.uint8)
        self.workspace = e(most(lambda N, K, F: max(
            B.bigcn_rms_norm_backward_workspace_bytes(N, K),
            B.bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F), 1)), dtype=torch.uint8)


def _fp4_bytes(rows, cols):
    groups = (cols + 31) // 32
    return rows * (groups * 16 + (groups + 3) // 4 * 4)


def _fp4_views(buf, rows, cols):
    """(q, exps) of 4-bit rows within a buffer."""
    groups = (cols + 31) // 32
    at, wide = rows * groups * 16, (groups + 3) // 4 * 4
    q = buf[:at].view(rows, groups * 16)[:, :(cols + 1) // 2]
    return q, buf[at:at + rows * wide].view(rows, wide)[:, :groups]


class ResidualLayer:
    """One layer of a residual stack in training:

        S = R + X (the stream with the previous layer's output added, in R's place),
        Y = gamma shat, shat the rows of S over their root mean square,
        H = A~ (Y4 W4 + b),

    Y4 and W4 the normalised rows and the weights' columns in microscaled 4 bits. A stack feeds each
    layer's H to the next as X and keeps one stream R; the first layer has none (S = X). Between
    ``forward()`` and ``backward()`` a layer keeps shat's 8-bit checkpoint and each row's rstd.

        G   = A~ dH                                       (the CSR is symmetric)
        dW  = (gamma v)^T G,   db = sum_i G_i             (v the checkpoint; straight through Y4 and W4)
        dY  = G4 W4r^T                                    (G's rows and W's rows in 4 bits)
        dX  = the norm's gradient of dY, plus dS          (of X and of R alike)

    In a stack dX is the dH and the dS of the layer below, which adds to it in place."""

    def __init__(self, N: int, K: int, F: int, device, eps: float = 1e-5, scratch=None):
        self.N, self.K, self.F, self.eps = N, K, F, eps
        self.device = torch.device(device)
        e = lambda *shape: torch.empty(shape, dtype=torch.float32, device=self.device)
        # parameters
        self.W, self.b = e(K, F), torch.zeros(F, device=self.device)
        self.gamma = torch.ones(K, device=self.device)
        # kept from forward to backward
        self.q, self.exps = B.checkpoint_buffers(N, K, self.device)
        self.rstd = e(N)
        self.H = e(N, F)
        # scratch: free for other layers between calls (dX until the layer below has run)
        scratch = scratch or ResidualScratch([(N, K, F)], self.device)
        take = lambda t, cols: t[:N * cols].view(N, cols)
        self.Y, self.Z, self.dX = take(scratch.Y, K), take(scratch.Z, F), take(scratch.dX, K)
        self.G, self.dY = self.Z, self.Y
        self.y4, self.g4 = _fp4_views(scratch.rows4, N, K), _fp4_views(scratch.rows4, N, F)
        self.w4 = _fp4_views(scratch.weights4, F, K)
        self.w4_rows = _fp4_views(scratch.weights4, K, F)
        self.workspace = scratch.workspace
        # gradients
        self.dW, self.db, self.dgamma = e(K, F), e(F), e(K)

    def forward(self, X, rowptr, colidx, R=None, S=None):
        """H from X (N x K fp32) and the stream R, to which X is added in place (or into S)."""
        S = R if S is None else S
        B.bigcn_rms_norm_forward(X, self.gamma, self.eps, R=R, S=S, Y=self.Y, rstd=self.rstd,
                                 q=self.q, exps=self.exps)
        B.bigcn_fp4_pack(self.Y, *self.y4)
        B.bigcn_fp4_pack_columns(self.W, *self.w4)
        B.bigcn_fp4_gemm(*self.y4, *self.w4, self.K, self.Z, bias=self.b)
        B.bigcn_spmm_norm(rowptr, colidx, self.Z, self.H)
        return self.H

    def backward(self, dH, rowptr, colidx, dS=None):
        """The gradients (dW, db, dgamma, dX) from dH = dL/dH (N x F) and, where the stream goes on
        behind this layer, dS = dL/dS by that way (N x K), in whose place dX then comes."""
        B.bigcn_spmm_norm(rowptr, colidx, dH, self.G)
        B.bigcn_checkpoint_weight_grad(self.q, self.exps, self.G, self.workspace, self.dW,
                                       gamma=self.gamma, db=self.db)
        B.bigcn_fp4_pack(self.G, *self.g4)
        B.bigcn_fp4_pack(self.W, *self.w4_rows)
        B.bigcn_fp4_gemm(*self.g4, *self.w4_rows, self.F, self.dY)
        dX = self.dX if dS is None else dS
        B.bigcn_rms_norm_backward(self.dY, self.gamma, self.rstd, self.workspace, q=self.q,
                                  exps=self.exps, dS=dS, dX=dX, dgamma=self.dgamma)
        return self.dW, self.db, self.dgamma, dX

    def gradients(self):
        """The parameters' gradients, in the order W, b, gamma."""
        return [self.dW, self.db, self.dgamma]


class GradientClip:
    """Scales the parameters' gradients of ``layers`` (anything whose ``gradients()`` lists them), in place,
    to at most a norm of all together; ``norm`` holds what it was. Their buffers are looked up once."""

    def __init__(self, layers):
        self.list = B.TensorList([t for layer in layers for t in layer.gradients()])
        device = self.list.tensors[0].device
        self.norm = torch.empty(1, dtype=torch.float32, device=device)
        self.workspace = torch.empty(B.bigcn_grad_norm_workspace_bytes(self.list), dtype=torch.uint8,
                                     device=device)

    def __call__(self, max_norm):
        B.bigcn_clip_grad_norm(self.list, max_norm, self.norm, self.workspace)
        return self.norm
