"""The kernels of the reading operators that only calls of some sizes choose, where the other tests' sizes choose another:
many rows of log probabilities in chunks, wide and narrow workgroups of attention with every part of a call."""

import numpy as np
import pytest
import torch

from oracle import reading as oracle
from paper_2106_12736_amd import sequence as seq
from test_gpu_reading import Make, attention_case, host, i32, within

pytestmark = pytest.mark.gpu


def rows_of(kind, R, V, m):
    v = torch.arange(V, device="cuda")
    if kind == "random":
        return m.act(R, V, scale=2.0)
    row = {"rising": v / 64.0, "falling": -v / 64.0, "equal": v * 0.0, "few": (v * 7 % 5).float(),
           "last": torch.where(v >= V - 3, 1.0, 0.0), "masked": torch.where(v % 3 == 1, v % 11 * 0.25, -float("inf")),
           "nan": torch.where(v == V - 2, float("nan"), v % 13 * 0.5)}[kind]
    return row.to(m.dtype).expand(R, V).contiguous()


@pytest.mark.parametrize("kind", ["random", "rising", "falling", "equal", "few", "last", "masked", "nan"])
@pytest.mark.parametrize("dtype,V,K", [("f32", 9001, 20), ("bf16", 17003, 128), ("f16", 30011, 1), ("bf16", 8193, 64)])
def test_many_rows_in_chunks(dtype, V, K, kind):
    R = 1100
    print(f"chunks {dtype} V={V} K={K} {kind}", flush=True)
    m = Make(V, dtype)
    z, tokens = rows_of(kind, R, V, m), m.ints(0, V, R)
    some = [0, 1, 700, R - 1]
    r = seq.token_logprobs_forward(z, tokens, top=K, temperature=0.9)
    logp, entropy, idx, top = oracle.token_logprobs(host(z[some]), tokens[some].cpu().numpy(), K, 0.9)
    # as in the tests of single rows: 1e-5 (1 + |ref|)
    for got, want, name in ((r.logp, logp, "logp"), (r.entropy, entropy, "entropy"), (r.top, top, "top")):
        within(got[some], want, 1e-5 * (1 + np.abs(np.where(np.isfinite(want), want, 0))), name)
    assert np.array_equal(r.idx[some].cpu().numpy(), idx)
    same = seq.token_logprobs_forward(z, tokens, temperature=0.9)
    within(same.entropy[some], entropy, 1e-5 * (1 + np.abs(np.where(np.isfinite(entropy), entropy, 0))), "entropy alone")
    if kind != "random":  # every row is the same
        assert torch.equal(r.idx, r.idx[:1].expand(R, K))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,Lq,Lk,H,G,D", [
    (1, 33, 65, 1, 1, 20),  # two waves a workgroup
    (2, 100, 150, 2, 2, 72),  # four
    (2, 250, 300, 2, 2, 48), (1, 260, 250, 2, 1, 100),  # eight, and their last tile in part
    (1, 4, 3000, 16, 2, 40), (3, 2, 20, 32, 2, 128), (1, 1, 9000, 1, 1, 8),  # few rows, in runs and not
])
def test_attention_forms(B, Lq, Lk, H, G, D, dtype):
    q_lengths = [Lq, Lq // 2, 1][:B]
    attention_case(B, Lq, Lk, H, G, D, dtype, q_lengths, [Lk - 1, Lk // 3, 0][:B], 0.7, seed=Lq)


def test_few_rows_of_every_number():
    m = Make(1, "bf16")
    k, v = m.act(2, 100, 1, 32), m.act(2, 100, 1, 32)
    for H in range(1, 34):
        q = m.act(2, H, 32)
        print(f"few rows H={H}", flush=True)
        want, _ = oracle.cross_attention(host(q)[:, None], host(k), host(v))
        within(seq.cross_attention_step(q, k, v), want[:, 0], (2.0 ** -8 + 2e-5) * np.abs(host(v)).max(), "y")


def test_outputs_given():
    m = Make(2, "bf16")
    q, k, v = m.act(2, 9, 4, 16), m.act(2, 20, 2, 16), m.act(2, 20, 2, 16)
    y, _ = seq.cross_attention_forward(q, k, v)
    wide = torch.full((2, 9, 4, 40), 7.0, dtype=torch.bfloat16, device="cuda")
    out, _ = seq.cross_attention_forward(q, k, v, y=wide[..., 8:24])
    assert torch.equal(out, y) and (wide[..., :8] == 7).all() and (wide[..., 24:] == 7).all()
    f, pos = m.f32(4).abs(), m.ints(0, 50, 2, 9, 1)
    turned = seq.rotary_forward(q, pos, f, y=wide[..., 20:36])
    assert torch.equal(turned, seq.rotary_forward(q, pos, f)) and (wide[..., 36:] == 7).all()
    z = m.act(3, 70)
    r = seq.token_logprobs_forward(z, i32([1, 2, 3]))
    rows = torch.full((3, 90), 7.0, dtype=torch.bfloat16, device="cuda")
    g = m.f32(3)
    gz = seq.token_logprobs_backward(r.stats, z, i32([1, 2, 3]), glogp=g, gz=rows[:, 10:80])
    assert torch.equal(gz, seq.token_logprobs_backward(r.stats, z, i32([1, 2, 3]), glogp=g))
    assert (rows[:, :10] == 7).all() and (rows[:, 80:] == 7).all()


def test_types():
    m = Make(3)
    q = m.f32(1, 2, 1, 8)
    with pytest.raises(ValueError, match="k must be"):
        seq.cross_attention_forward(q, q.half(), q)
    with pytest.raises(ValueError, match="must be float32, bfloat16 or float16"):
        seq.cross_attention_forward(q.double(), q.double(), q.double())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
@pytest.mark.parametrize("Lk", [60, 150, 300])
def test_every_workgroup_of_attention(Lk, D, dtype):
    # two, four and eight waves, of rows and of keys, over several tiles in one run and in several
    attention_case(2, 150, Lk, 4, 2, D, dtype, lengths=[Lk, Lk - 7], seed=D)
    attention_case(40, 130, Lk, 8, 8, D, dtype, seed=Lk)
    attention_case(2, 60, Lk, 2, 2, D, dtype, [60, 31], seed=D + Lk)
