"""The weight gradient's runs of rows, added by its second kernel from the workspace: a run whose
CTA gave up (its bounded waits ran out) shows as NaN in every sum that lacks its rows, whatever the
workspace held before. The probe abandons a run as the first kernel does; no wait is made to run out."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from norm_reference import U
from paper_2010_07565_gb300 import build as lib_build
from test_gpu_norm import f64, rng, within

PROBE = os.path.join(os.path.dirname(__file__), "probes", "grad_runs.cu")

# K, F, NT, tiles of a group, runs of a full group, runs of the last
LAYOUTS = [(70, 9, 64, 1, 5, 5), (300, 100, 64, 2, 3, 2), (640, 200, 128, 2, 70, 34),
           (1300, 300, 256, 1, 9, 9), (520, 256, 256, 1, 38, 38)]


@pytest.fixture(scope="module")
def add_runs(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("probe") / "grad_runs.so")
    subprocess.run([lib_build.nvcc(), *lib_build.ARCH, "-O3", "-std=c++17", "--expt-relaxed-constexpr",
                    "-I", lib_build.INCLUDE, "-I", lib_build.CSRC, "-shared", "-Xcompiler", "-fPIC",
                    "-o", so, PROBE], check=True)
    f = ctypes.CDLL(so).add_runs
    p, i, l = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    f.argtypes, f.restype = [p, p, l, l, i, i, i, i, i, i, i, p, p, p, p, i, i, i], i
    return f


@pytest.mark.gpu
@pytest.mark.parametrize("affine", [False, True])
@pytest.mark.parametrize("K,F,NT,mt,full,last", LAYOUTS)
def test_an_abandoned_run_is_nan(cuda_device, add_runs, K, F, NT, mt, full, last, affine):
    tiles = -(-K // 128)
    groups, nt = -(-tiles // mt), -(-F // NT)
    runs = lambda g: last if g == groups - 1 else full
    r = rng(K + F)
    # What an earlier call left: plausible sums in every place.
    partial = r.standard_normal((nt, tiles, full, NT, 128)).astype(np.float32)
    colsum = r.standard_normal((full, nt * NT)).astype(np.float32)
    gamma, beta = r.standard_normal(K).astype(np.float32), r.standard_normal(K).astype(np.float32)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    dgamma, dbeta = (t(gamma), t(beta)) if affine else (None, None)
    dW, db = torch.empty((K, F), device=cuda_device), torch.empty(F, device=cuda_device)

    def call(group, run, ny):
        w, c = t(partial), t(colsum)
        dW.fill_(7.0), db.fill_(7.0)
        a = [x.data_ptr() if x is not None else None for x in (dgamma, dbeta)]
        assert add_runs(w.data_ptr(), c.data_ptr(), tiles, groups, full, last, mt, NT, nt, K, F, *a,
                        dW.data_ptr(), db.data_ptr(), group, run, ny) == 0
        return f64(w), f64(c)

    # All there: the sums of the runs, at most 2 x 70 + 16 fp32 additions each.
    col_group = np.arange(F) % NT // 64
    cs = np.array([colsum[:runs(col_group[j]), j].astype(np.float64).sum() for j in range(F)])
    ca = np.array([np.abs(colsum[:runs(col_group[j]), j]).sum() for j in range(F)])
    sums, size = np.empty((K, F)), np.empty((K, F))
    for k in range(K):
        part = partial[:, k // 128, :runs(k // 128 // mt), :, k % 128].astype(np.float64)
        sums[k] = part.sum(1).reshape(-1)[:F]
        size[k] = np.abs(part).sum(1).reshape(-1)[:F]
    g, b = (gamma[:, None], beta[:, None]) if affine else (np.ones((K, 1)), np.zeros((K, 1)))
    ref, bound = g * sums + b * cs, 160 * U * (np.abs(g) * size + np.abs(b) * ca)
    call(-1, 0, 0)
    within(dW, ref, bound, "dW")
    within(db, cs, 160 * U * ca, "db")

    # A run abandoned: NaN in the group's features times the column tile, and in the columns that
    # the group sums; everything else as before. Nothing else of the workspace is touched.
    for group in {0, groups // 2, groups - 1}:
        for run in {0, runs(group) - 1}:
            for ny in {0, nt - 1}:
                w, c = call(group, run, ny)
                bad_w = np.zeros(partial.shape, bool)
                bad_w[ny, group * mt:(group + 1) * mt, run] = True
                own = [j for j in range(F) if j // NT == ny and col_group[j] == group]
                bad_c = np.zeros(colsum.shape, bool)
                bad_c[run, own] = True
                assert np.array_equal(np.isnan(w), bad_w) and np.array_equal(w[~bad_w], partial[~bad_w])
                assert np.array_equal(np.isnan(c), bad_c) and np.array_equal(c[~bad_c], colsum[~bad_c])
                bad = np.zeros((K, F), bool)
                bad[group * mt * 128:(group + 1) * mt * 128, ny * NT:(ny + 1) * NT] = True
                if affine:
                    bad[:, own] = True
                assert np.array_equal(np.isnan(f64(dW)), bad)
                within(f64(dW)[~bad], ref[~bad], bound[~bad], "dW")
                fine = [j for j in range(F) if j not in own]
                assert np.isnan(f64(db)[own]).all()
                within(f64(db)[fine], cs[fine], 160 * U * ca[fine], "db")
