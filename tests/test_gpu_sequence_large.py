"""Tensors of more than 2^31 elements: the sequence operators' last rows, whose offsets pass 32 bits, against
the float64 oracle on those rows alone (tolerances as in test_gpu_sequence)."""

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from oracle import sequence as oracle
from paper_2106_12736_amd import sequence as seq
from test_gpu_sequence import check, host

pytestmark = pytest.mark.gpu

B16 = torch.bfloat16


def _act(*shape, scale=1.0):
    assert torch.Size(shape).numel() > 2 ** 31
    return torch.empty(shape, dtype=B16, device="cuda").normal_(std=scale)


@pytest.fixture(autouse=True)
def _seeded():
    torch.manual_seed(0)
    yield
    torch.cuda.empty_cache()


def test_conv_past_32_bits():
    L, D, n = 66000, 32800, 4
    x, gy = _act(1, L, D), _act(1, L, D)
    w, b = torch.randn(D, n, device="cuda"), torch.randn(D, device="cuda")
    print("conv", x.shape, flush=True)
    y, _ = seq.causal_conv_forward(x, w, bias=b, silu=True)
    gx, gw, _ = seq.causal_conv_backward(gy, x, w, bias=b, silu=True)
    d = [0, 5, D - 1]
    cut = lambda t: host(t[:, -40:, d])  # noqa: E731
    ry, _ = oracle.causal_conv(cut(x), host(w[d]), host(b[d]), True)
    check(y[:, -30:, d], ry[:, -30:], "y")
    rx, _, _ = oracle.causal_conv_backward(cut(gy), cut(x), host(w[d]), host(b[d]), True)
    check(gx[:, -30:, d], rx[:, -30:], "gx")
    assert bool(torch.isfinite(gw).all())


def test_scan_past_32_bits():
    L, D, N = 66000, 32800, 2
    x, dt, gy = _act(1, L, D), _act(1, L, D, scale=0.1), _act(1, L, D)
    A = torch.full((D, N), -8.0, device="cuda")  # steps of about 0.7: 40 tokens leave nothing of a state
    Bm, Cm = (torch.randn(1, L, 1, N, device="cuda").to(B16) for _ in range(2))
    print("scan", x.shape, flush=True)
    y, h, saved = seq.scan_forward(x, dt, A, Bm, Cm, last=True, save=True)
    g = seq.scan_backward(gy, saved, x, dt, A, Bm, Cm)
    d = [0, 7, D - 1]
    v = [host(x[:, -80:, d]), host(dt[:, -80:, d]), host(A[d]), host(Bm[:, -80:]), host(Cm[:, -80:])]
    ry, rh, _ = oracle.scan(*v)
    check(y[:, -30:, d], ry[:, -30:], "y")
    check(h[:, d], rh, "h")
    want = oracle.scan_backward(host(gy[:, -80:, d]), *v)
    check(g.x[:, -30:, d], want["x"][:, -30:], "gx")
    check(g.dt[:, -30:, d], want["dt"][:, -30:], "gdt")


def test_norm_past_32_bits():
    R, D = 530000, 4096
    x, f, gout = _act(R, D), _act(R, D), _act(R, D)
    w = [torch.randn(D, device="cuda") for _ in range(3)]
    print("norm", x.shape, flush=True)
    out, n, stats = seq.block_norm_forward(x, f, scale=w[0], w_post=w[1], w_pre=w[2])
    g = seq.block_norm_backward(gout, x, stats, x, f, scale=w[0], w_post=w[1], w_pre=w[2])
    hx, hf, hw = host(x[-3:]), host(f[-3:]), [host(t) for t in w]
    rout, rn = oracle.block_norm(hx, hf, None, *hw)
    check(out[-3:], rout, "out")
    check(n[-3:], rn, "n")
    want = oracle.block_norm_backward(host(gout[-3:]), hx, hx, hf, None, *hw)
    check(g.x[-3:], want["x"], "gx")
    check(g.f[-3:], want["f"], "gf")


@pytest.mark.parametrize("R,V", [(40000, 60000), (20000, 120000)])  # rows in registers, rows in segments
def test_distill_past_32_bits(R, V):
    z = _act(R, V, scale=2.0)
    idx = torch.randint(0, V, (R, 4), device="cuda", dtype=torch.int32)
    teacher, gloss = torch.randn(R, 4, device="cuda").to(B16), torch.randn(R, device="cuda")
    print("distill", z.shape, flush=True)
    last = z[-2:].clone()
    loss, gz = seq.distill_forward_backward(gloss, z, idx, teacher, temperature=1.5, gz=z)
    rloss, rgz = oracle.distill(host(last), idx[-2:].cpu().numpy(), host(teacher[-2:]), 1.5, gloss=host(gloss[-2:]))
    check(loss[-2:], rloss, "loss")
    for r in range(2):
        check(gz[r - 2], rgz[r], "gz")
