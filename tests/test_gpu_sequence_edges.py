"""The sequence operators on values and layouts at the edge of what they take, and on the kernels that only
larger calls reach, against the float64 oracle (tolerances as in test_gpu_sequence)."""

import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from oracle import sequence as oracle
from paper_2106_12736_amd import sequence as seq
from test_gpu_sequence import Make, check, host

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------
# block norm
# ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [7, 96, 5000])
@pytest.mark.parametrize("gout", [False, True])
def test_norm_gradients_of_large_rows(dtype, D, gout):
    # the reciprocal root mean square cubed is past float32's range for these rows, the gradient is not
    print(f"norm large rows D={D} {dtype} gout={gout}", flush=True)
    m = Make(D, dtype)
    sizes = [1.0, 1e10, 1e13, 1e14, 1e15]
    x, f, gn = (m.act(len(sizes), D) for _ in range(3))
    for r, s in enumerate(sizes):
        x[r] *= s
        f[r] *= s
    w = [m.f32(D, mean=1.0, scale=0.3) for _ in range(2)]
    # out of the size of x: f is normed; and out of the size of f: it is not
    for w_post in (w[0], None):
        _, _, stats = seq.block_norm_forward(x, f, w_post=w_post, w_pre=w[1])
        go = (m.act(len(sizes), D).float() / torch.tensor(sizes, device="cuda")[:, None]).to(x.dtype) if gout else None
        g = seq.block_norm_backward(go, gn, stats, x, f, w_post=w_post, w_pre=w[1])
        want = oracle.block_norm_backward(host(go), host(gn), host(x), host(f), w_post=host(w_post), w_pre=host(w[1]))
        for r in range(len(sizes)):
            check(g.x[r], want["x"][r], f"gx {r}")
            check(g.f[r], want["f"][r], f"gf {r}")


@pytest.mark.parametrize("D", [1, 64, 5000])
def test_norm_rows_of_zeros_under_a_small_eps(D):
    print(f"norm zeros D={D}", flush=True)
    m = Make(D)
    x, f, gout, gn = (m.act(3, D) for _ in range(4))
    x[0] = f[0] = 0
    w = torch.ones(D, device="cuda")
    eps = float(np.float32(1e-28))
    _, _, stats = seq.block_norm_forward(x, f, w_post=w, w_pre=w, eps=eps)
    g = seq.block_norm_backward(gout, gn, stats, x, f, w_post=w, w_pre=w, eps=eps)
    want = oracle.block_norm_backward(host(gout), host(gn), host(x), host(f), w_post=host(w), w_pre=host(w), eps=eps)
    # of a single channel the gradient is the eps itself, times 1e14 where the row is 0 and below 1e-20 elsewhere
    for r in range(3 if D > 1 else 1):
        check(g.x[r], want["x"][r], f"gx {r}")
        check(g.f[r], want["f"][r], f"gf {r}")
