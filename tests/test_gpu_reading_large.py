"""The reading operators past 32-bit offsets: tensors of more than 2^31 elements, checked where the far ones lie."""

import numpy as np
import pytest
import torch

from oracle import reading as oracle
from paper_2106_12736_amd import sequence as seq

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def host(t):
    return t.detach().double().cpu().numpy()


@pytest.fixture(autouse=True)
def free():
    yield
    torch.cuda.empty_cache()


def test_rotary_far_tokens():
    B, L, H, D = 1, 280_000, 64, 128
    print(f"rotary {B * L * H * D} elements", flush=True)
    x = torch.zeros(B, L, H, D, dtype=BF16, device="cuda")
    x[:, -5:] = torch.randn(5, H, D, device="cuda").to(BF16)
    pos = torch.arange(L, device="cuda", dtype=torch.int32)[None, :, None].contiguous()
    f = 10000.0 ** (-torch.arange(64, device="cuda") / 64.0)
    y = seq.rotary_forward(x, pos, f)
    want = oracle.rotary(host(x[:, -5:]), pos[:, -5:].cpu().numpy(), host(f))
    # a rounding, and 1e-6 of the largest value
    assert (np.abs(host(y[:, -5:]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-5).all()
    assert torch.count_nonzero(y[:, :-5]) == 0


@pytest.mark.parametrize("Lq,H", [(1, 4), (70, 2)])
def test_attention_far_keys(Lq, H):
    B, Lk, G, D = 2, 9_000_000, 1, 128
    print(f"attention {B * Lk * G * D} elements of k, Lq={Lq} H={H}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(Lq)
    k, v = (torch.full((B, Lk, G, D), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
    at = torch.tensor([0, 3, 4_499_999, Lk - 70, Lk - 2, Lk - 1], device="cuda")
    mask = torch.zeros(B, Lk, dtype=torch.bool, device="cuda")
    mask[:, at] = True
    for t in (k, v):
        t[:, at] = torch.randn(B, len(at), G, D, generator=g, device="cuda").to(BF16)
    q, gy = (torch.randn(B, Lq, H, D, generator=g, device="cuda").to(BF16) for _ in range(2))
    y, saved = seq.cross_attention_forward(q, k, v, mask=mask, save=True)
    hk, hv = host(k[:, at]), host(v[:, at])
    want, _ = oracle.cross_attention(host(q), hk, hv)
    # roundings of six probabilities and of y, u each, on values up to 5
    assert (np.abs(host(y) - want) <= 2.0 ** -8 * (np.abs(want) + np.abs(hv).max())).all()
    grads = seq.cross_attention_backward(gy, y, saved, q, k, v, mask=mask)
    for got, ref, name in zip((grads.q, grads.k[:, at], grads.v[:, at]),
                              oracle.cross_attention_backward(host(gy), host(q), hk, hv), ("gq", "gk", "gv")):
        # relative to the whole: a rounding of a factor and one of the result, 2^-8 each, and delta's
        off = np.linalg.norm(host(got) - ref) / np.linalg.norm(ref)
        assert off <= 3 * 2.0 ** -8, (name, off)
    for t in grads[1:]:
        t[:, at] = 0
        assert torch.count_nonzero(t) == 0


def test_logprobs_far_rows():
    R, V, K = 20_000, 120_000, 8
    print(f"logprobs {R * V} logits", flush=True)
    z = torch.zeros(R, V, dtype=BF16, device="cuda")
    some = [0, 17_895, 17_896, R - 1]
    z[some] = (torch.randn(len(some), V, device="cuda") * 2).to(BF16)
    tokens = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    tokens[some] = torch.tensor([5, V - 1, 0, V - 1], dtype=torch.int32, device="cuda")
    glogp = torch.zeros(R, device="cuda")
    glogp[some] = 1.0
    r = seq.token_logprobs_forward(z, tokens, top=K)
    logp, entropy, idx, top = oracle.token_logprobs(host(z[some]), tokens[some].cpu().numpy(), K)
    for got, want in ((r.logp, logp), (r.entropy, entropy), (r.top, top)):
        assert (np.abs(host(got[some]) - want) <= 1e-5 * (1 + np.abs(want))).all()
    assert np.array_equal(r.idx[some].cpu().numpy(), idx)
    assert torch.equal(r.idx[1:100], torch.arange(K, dtype=torch.int32, device="cuda").expand(99, K))
    gz = seq.token_logprobs_backward(r.stats, z, tokens, glogp=glogp, gz=z)
    # a row's gradient sums to nothing: 1 at the token less probabilities that add up to 1, each rounded
    for i in some:
        assert abs(float(gz[i].double().sum())) <= 2.0 ** -8
        assert float(gz[i, tokens[i]]) > 0.5
    gz[some] = 0
    assert torch.count_nonzero(gz) == 0


def test_rotary_more_threads_than_a_launch_has():
    # 2^31 tokens of 5 heads: with 4 heads a thread a launch of 2^32 threads, so all 5
    B, L, H = 8, 1 << 28, 5
    print(f"rotary {B * L * H * 2} elements", flush=True)
    x = torch.zeros(B, L, H, 2, dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, L // 2 - 1, L // 2, L - 2, L - 1], device="cuda")
    x[:, at] = torch.randn(B, len(at), H, 2, device="cuda").to(BF16)
    pos = torch.arange(L, device="cuda", dtype=torch.int32)[:, None].contiguous()
    f = torch.tensor([0.37], device="cuda")
    want = oracle.rotary(host(x[:, at]), pos[at].cpu().numpy(), host(f))
    assert seq.rotary_forward(x, pos, f, y=x) is x
    # a rounding, and 1e-6 of the largest value
    assert (np.abs(host(x[:, at]) - want) <= 2.0 ** -8 * np.abs(want) + 1e-5).all()
