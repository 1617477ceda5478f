"""Pins of the oracle of the reading operators: closed forms, torch's functions, central differences."""

import numpy as np
import pytest
import torch

from oracle import reading as oracle

RNG = np.random.default_rng


def _differences(f, x, up, eps=1e-6):
    """Gradient of sum(up * f(x)) by central differences."""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = (up * (f(a) - f(b))).sum() / (2 * eps)
    return g


# ---- rotary ----------------------------------------------------------------------
def test_rotary_quarter_turn():
    x = np.array([1.0, 2.0, 3.0, 4.0, 5.0]).reshape(1, 1, 1, 5)
    f = np.array([np.pi / 2, np.pi])
    got = oracle.rotary(x, np.array([[[1]]]), f)  # pairs (0, 2) and (1, 3)
    assert np.allclose(got[0, 0, 0], [-3, -2, 1, -4, 5], atol=1e-12)
    got = oracle.rotary(x, np.array([[[1]]]), f, interleaved=True)
    assert np.allclose(got[0, 0, 0], [-2, 1, -3, -4, 5], atol=1e-12)


def test_rotary_products_depend_on_the_distance():
    rng = RNG(0)
    q, k, f = rng.standard_normal((1, 1, 1, 8)), rng.standard_normal((1, 1, 1, 8)), rng.random(4)
    at = lambda x, t, h: oracle.rotary(x, np.array([[[t, h]]]), f, (1, 3))  # noqa: E731
    a = (at(q, 7, 5) * at(k, 3, 9)).sum()
    assert np.isclose(a, (at(q, 107, 45) * at(k, 103, 49)).sum())
    assert not np.isclose(a, (at(q, 8, 5) * at(k, 3, 9)).sum())


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_backward_is_its_adjoint(interleaved):
    rng = RNG(1)
    x, gy = rng.standard_normal((2, 2, 5, 3, 11))
    pos, f, n = rng.integers(0, 100, (2, 5, 2)), rng.random(4), [3, 5]
    kw = dict(sections=(1, 3), interleaved=interleaved, lengths=n)
    y, gx = oracle.rotary(x, pos, f, **kw), oracle.rotary(gy, pos, f, inverse=True, **kw)
    live = np.arange(5)[None, :, None, None] < np.array(n)[:, None, None, None]
    assert np.isclose((y * gy * live).sum(), (x * gx * live).sum())
    assert not y[0, 3:].any() and not gx[0, 3:].any()
    assert np.allclose(oracle.rotary(y, pos, f, inverse=True, **kw), x * live)


# ---- attention ---------------------------------------------------------------------
def test_attention_against_torch():
    rng = RNG(2)
    q, gy = rng.standard_normal((2, 2, 4, 6, 5))
    k, v = rng.standard_normal((2, 2, 7, 3, 5))
    mask = rng.random((2, 7)) < 0.6
    mask[:, 0] = True
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    heads = lambda t: t.transpose(1, 2)  # noqa: E731
    each = lambda t: heads(t).repeat_interleave(2, 1)  # noqa: E731
    out = heads(torch.nn.functional.scaled_dot_product_attention(
        heads(tq), each(tk), each(tv), attn_mask=torch.tensor(mask)[:, None, None], scale=0.7))
    y, lse = oracle.cross_attention(q, k, v, 0.7, mask=mask)
    assert np.allclose(y, out.detach().numpy())
    s = torch.where(torch.tensor(mask)[:, None, None], heads(tq) @ each(tk).transpose(-1, -2) * 0.7, -torch.inf)
    assert np.allclose(lse, torch.logsumexp(s, -1).detach().numpy())
    for got, want in zip(oracle.cross_attention_backward(gy, q, k, v, 0.7, mask=mask),
                         torch.autograd.grad(out, (tq, tk, tv), torch.tensor(gy))):
        assert np.allclose(got, want.numpy())


def test_attention_backward_against_differences():
    rng = RNG(3)
    q, k, v = rng.standard_normal((2, 3, 2, 3)), rng.standard_normal((2, 4, 1, 3)), rng.standard_normal((2, 4, 1, 3))
    gy = rng.standard_normal(q.shape)
    kw = dict(scale=0.9, q_lengths=[2, 3], lengths=[4, 3], mask=np.array([[1, 0, 1, 1], [0, 1, 1, 1]]))
    f = lambda q=q, k=k, v=v: oracle.cross_attention(q, k, v, **kw)[0]  # noqa: E731
    got = oracle.cross_attention_backward(gy, q, k, v, **kw)
    for name, x, g in zip("qkv", (q, k, v), got):
        assert np.allclose(g, _differences(lambda t: f(**{name: t}), x, gy), atol=1e-7), name


def test_attention_nothing_to_read():
    q, k = np.ones((2, 3, 1, 2)), np.full((2, 4, 1, 2), np.nan)
    k[1, 2] = 1.0
    kw = dict(mask=np.array([[0, 0, 0, 0], [0, 0, 1, 0]]), q_lengths=[3, 1])
    y, lse = oracle.cross_attention(q, k, k, **kw)
    assert not y[0].any() and (lse[0] == -np.inf).all()
    assert (y[1, 0] == 1).all() and not y[1, 1:].any() and (lse[1, :, 1:] == -np.inf).all()
    gq, gk, gv = oracle.cross_attention_backward(q, q, k, k, **kw)
    assert not gq.any() and not gk.any() and (gv[1, 2] == 1).all() and gv.sum() == 2


# ---- log probabilities -----------------------------------------------------------------
def test_logprobs_against_torch():
    rng = RNG(4)
    z, tokens = rng.standard_normal((5, 9)), np.array([3, 0, -1, 8, 2])
    glogp, gentropy, gtop = rng.standard_normal(5), rng.standard_normal(5), rng.standard_normal((5, 3))
    tz = torch.tensor(z, requires_grad=True)
    l = torch.log_softmax(tz / 0.7, 1)
    logp, entropy, idx, values = oracle.token_logprobs(z, tokens, 3, 0.7)
    mine = torch.where(torch.tensor(tokens) >= 0, l.gather(1, torch.tensor(tokens).clamp(min=0)[:, None])[:, 0], 0.0)
    h = -(l.exp() * l).sum(1)
    tops = l.topk(3, 1)
    assert np.allclose(logp, mine.detach()) and np.allclose(entropy, h.detach())
    assert np.array_equal(idx, tops.indices) and np.allclose(values, tops.values.detach())
    want = torch.autograd.grad([mine, h, tops.values], tz, [torch.tensor(g) for g in (glogp, gentropy, gtop)])[0]
    assert np.allclose(oracle.token_logprobs_backward(z, tokens, glogp, gentropy, idx, gtop, 0.7), want)


def test_logprobs_backward_against_differences():
    rng = RNG(5)
    z, tokens, gentropy = rng.standard_normal((3, 6)), np.array([1, 5, -1]), rng.standard_normal(3)
    want = _differences(lambda t: np.stack(oracle.token_logprobs(t, tokens, 0, 1.3)[:2]), z, np.stack([np.ones(3), gentropy]))
    assert np.allclose(oracle.token_logprobs_backward(z, tokens, np.ones(3), gentropy, temperature=1.3), want, atol=1e-8)


def test_logprobs_edges():
    inf = np.inf
    z = np.array([[0, 0, 0, 0.0], [1, -inf, 1, -inf], [-inf] * 4, [2, np.nan, 3, np.nan], [0, -0.0, 1, 0.0], [1, inf, 0, 0]])
    logp, entropy, idx, values = oracle.token_logprobs(z, [0, 1, 2, 0, 9, 0], 3)
    assert np.allclose(entropy[:2], [np.log(4), np.log(2)]) and np.isnan(entropy[[2, 3, 5]]).all()
    assert np.isclose(logp[0], -np.log(4)) and logp[1] == -inf and np.isnan(logp[2:]).all()
    assert idx.tolist() == [[0, 1, 2], [0, 2, 1], [0, 1, 2], [1, 3, 2], [2, 0, 1], [1, 0, 2]]
    gz = oracle.token_logprobs_backward(z[:2], [0, 9], np.ones(2))
    assert np.allclose(gz[0], [0.75, -0.25, -0.25, -0.25]) and np.isnan(gz[1]).all()
    assert not oracle.token_logprobs_backward(z, [0, 1, 2, 0, 9, 0], np.zeros(6)).any()
    # a place of -inf takes no part in the entropy's gradient
    assert np.allclose(oracle.token_logprobs_backward(z[1:2], gentropy=np.ones(1)), 0)
