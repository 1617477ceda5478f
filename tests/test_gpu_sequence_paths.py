"""The kernels of the sequence operators that only larger calls choose, against the float64 oracle (tolerances as in
test_gpu_sequence): the scan's step for four sequences a thread, the distillation's rows in registers with masks
and places out of range, and the block norm's second and later rows of a workgroup in each of its widths."""

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from oracle import sequence as oracle
from paper_2106_12736_amd import sequence as seq
from test_gpu_sequence import Make, check, distill_case, host, norm_case, scan_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,G,least", [(5, 1, 63), (8, 4, 63), (16, 2, 32), (30, 1, 16), (64, 2, 8)])
@pytest.mark.parametrize("more", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_step_of_many_sequences(N, G, least, more, dtype):
    # four sequences a thread from 2048 workgroups of one: every remainder of the sequences by 4, a last
    # workgroup that is not full, each number of lanes a channel
    B, D = least + more, 4100
    print(f"scan step B={B} D={D} N={N} G={G} {dtype}", flush=True)
    m = Make(N + more, dtype)
    v = scan_inputs(m, B, None, D, N, G, True, True, True, True, None, "dense")
    h = m.f32(B, D, N)
    token = ("x", "dt", "B", "C", "gate")
    ry, rh, _ = oracle.scan(**{k: host(t[:, None] if k in token else t) for k, t in v.items()}, h0=host(h))
    y, new = seq.scan_step(**v, h=h, h_new=torch.empty_like(h))
    check(y, ry[:, 0], "y")
    check(new, rh, "h")
    inplace = h.clone()
    y2, same = seq.scan_step(**v, h=inplace)
    assert same is inplace and torch.equal(y, y2) and torch.equal(new, inplace)


@pytest.mark.parametrize("R,V", [(260, 60), (260, 301), (260, 7001), (260, 16001), (770, 20001), (770, 33000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_distill_masked_and_odd_rows_in_registers(R, V, dtype):
    lowest = {"f32": torch.finfo(torch.float32).min, "bf16": torch.finfo(torch.bfloat16).min, "f16": -65504.0}

    def change(v):
        z, idx, t = v["z"], v["idx"], v["teacher"]
        named = torch.cat([idx[1].long(), v["labels"][1:2].long()])
        free = torch.ones(V, dtype=torch.bool, device="cuda")
        free[named] = False
        free = free.nonzero()[:, 0]
        z[1, free[: V // 3]] = float("-inf")             # a vocabulary masked with -inf
        z[1, free[V // 3: V // 2]] = lowest[dtype]       # and with the type's lowest value
        z[2] = lowest[dtype]                             # everywhere
        t[3, :3] = float("-inf")                         # teacher entries of no probability
        idx[4, 1] = idx[4, 0]                            # one place given twice
        idx[5, 1:] = idx[5, 0]                           # one place alone
        v["labels"][5] = idx[5, 0]
        t[6] = float("-inf")                             # a teacher that says nothing
        idx[7, 2] = V                                    # an index past the vocabulary
        v["labels"][8] = V                               # a label past it
        z[9] = float("-inf")                             # a row of nothing at all
        z[10, free[0]] = float("nan")
        idx[11] = -1                                     # neither teacher nor label
        v["labels"][11] = -1

    distill_case(R, V, 8, dtype, tau=1.5, weight=False, holes=False, change=change, seed=V)
    distill_case(R, V, 8, dtype, tau=1.5, alpha=0.0, change=change, seed=V + 1)
    distill_case(R, V, 8, dtype, tau=0.7, alpha=1.0, change=change, seed=V + 2)


# rows of one wave, and of 2, 4, 8 and 16 with a vector or two a thread
@pytest.mark.parametrize("R,D,dtype", [(8500, 130, "bf16"), (4500, 700, "bf16"), (2500, 1500, "bf16"), (1200, 3000, "bf16"),
                                       (700, 8000, "bf16"), (700, 4500, "f16"), (8500, 70, "f32"), (4500, 400, "f32"),
                                       (2500, 1001, "f32"), (1200, 2000, "f32"), (700, 4000, "f32"), (700, 5001, "f32")])
def test_norm_many_rows(R, D, dtype):
    norm_case(R, D, dtype=dtype, seed=R + D)
