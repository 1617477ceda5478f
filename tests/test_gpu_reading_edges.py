"""The reading operators at values and sizes that could go wrong without another test's seeing it.

Infinities and NaN in keys and values that a sequence's queries see, beside rows past its queries: those rows' outputs and
gradients are 0, and so are the gradients of keys that no query reads.  What the rows that read them get is the oracle's,
NaN and infinities at the same places; tolerances are those of the tests of finite values.
"""

import numpy as np
import pytest
import torch

from oracle import reading as oracle
from paper_2106_12736_amd import sequence as seq
from test_gpu_reading import UNIT, Make, bounds, host, i32, within

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")

FORMS = {"tiles": (3, 77, 130, 2, 2, 40), "keys in runs": (3, 40, 1500, 1, 1, 64), "wide": (3, 300, 70, 4, 2, 128),
         "few rows": (3, 4, 200, 4, 2, 32), "few rows in runs": (3, 4, 9000, 2, 1, 40), "rows in runs": (3, 700, 20, 2, 1, 24),
         "odd width": (3, 150, 65, 1, 1, 63)}


class Seen:
    """A call whose key Lk / 2 holds `value` in its last channel, in k or v (or k, and the next key's v -value); its sequences
    have no, some and all queries."""

    def __init__(self, form, dtype, where, value):
        B, Lq, Lk, H, G, D = FORMS[form]
        print(f"seen {form} {dtype} {where} {value}", flush=True)
        m = Make(Lq + D, dtype)
        self.q, self.k, self.v, self.gy = m.act(B, Lq, H, D), m.act(B, Lk, G, D), m.act(B, Lk, G, D), m.act(B, Lq, H, D)
        self.q[..., -1] = self.q[..., -1].abs() + 0.5  # a key of -inf there has a score of -inf with every query
        if where == "both":
            self.k[:, Lk // 2, :, -1], self.v[:, Lk // 2 + 1, :, -1] = value, -value
        else:
            (self.k if where == "k" else self.v)[:, Lk // 2, :, -1] = value
        self.n = [0, Lq // 2 + 1, Lq]
        for b, n in enumerate(self.n):
            self.q[b, n:], self.gy[b, n:] = NAN, INF
        self.kw = dict(q_lengths=i32(self.n))
        self.y, self.saved = seq.cross_attention_forward(self.q, self.k, self.v, save=True, **self.kw)

    def hosts(self):
        return host(self.q), host(self.k), host(self.v)

    def bounds(self, y):
        with np.errstate(all="ignore"):
            return bounds(host(self.gy), *self.hosts(), y, self.q.shape[-1] ** -0.5, self.n, None, None)

    def wanted(self):
        with np.errstate(all="ignore"):
            return oracle.cross_attention(*self.hosts(), q_lengths=self.n)

    def factor(self):
        """Half a step of what a 16-bit factor of a sum is rounded to."""
        return UNIT[self.y.dtype] if self.y.dtype != torch.float32 else 0.0


SEEN = [("k", NAN), ("k", -INF), ("v", INF), ("v", NAN), ("both", -INF)]


@pytest.mark.parametrize("where,value", SEEN)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS)
def test_rows_past_the_queries_are_zero(form, dtype, where, value):
    s = Seen(form, dtype, where, value)
    for b, n in enumerate(s.n):
        assert (s.y[b, n:] == 0).all(), b
    ry, rlse = s.wanted()
    (ay, _, _, _), _ = s.bounds(ry)
    within(s.y, ry, (s.factor() + 2e-5) * ay, "y")
    within(s.saved[:rlse.size].view(rlse.shape), rlse, 2e-5 * (1 + np.abs(np.where(np.isfinite(rlse), rlse, 0))), "lse")
    again, _ = seq.cross_attention_forward(s.q, s.k, s.v, **s.kw)
    assert torch.equal(again.nan_to_num(7.0), s.y.nan_to_num(7.0))


# the gradient of the queries
@pytest.mark.parametrize("where,value", SEEN)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS)
def test_gradients_past_the_queries_are_zero(form, dtype, where, value):
    s = Seen(form, dtype, where, value)
    g = seq.cross_attention_backward(s.gy, s.y, s.saved, s.q, s.k, s.v, **s.kw)
    for b, n in enumerate(s.n):
        assert (g.q[b, n:] == 0).all(), b
    ry, _ = s.wanted()
    (_, aq, _, _), (pq, _) = s.bounds(ry)
    with np.errstate(all="ignore"):
        want = oracle.cross_attention_backward(host(s.gy), *s.hosts(), q_lengths=s.n)[0]
        within(g.q, want, s.factor() * aq + 4e-5 * pq, "gq")


# the gradients of the keys and values
@pytest.mark.parametrize("where,value", SEEN)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("form", FORMS)
def test_gradients_of_keys_are_those_of_the_queries_there(form, dtype, where, value):
    s = Seen(form, dtype, where, value)
    g = seq.cross_attention_backward(s.gy, s.y, s.saved, s.q, s.k, s.v, **s.kw)
    assert (g.k[0] == 0).all() and (g.v[0] == 0).all()
    ry, _ = s.wanted()
    (_, _, ak, av), (_, pk) = s.bounds(ry)
    with np.errstate(all="ignore"):
        _, gk, gv = oracle.cross_attention_backward(host(s.gy), *s.hosts(), q_lengths=s.n)
        within(g.v, gv, (s.factor() + 2e-5) * av, "gv")
        if where == "k":
            within(g.k, gk, s.factor() * ak + 4e-5 * pk, "gk")
        else:  # infinite or NaN: a sum of infinities of both signs, and of what y's infinity leaves of delta
            assert not np.isfinite(gk[1:]).any() and not torch.isfinite(g.k[1:]).any()


# ----------------------------------------------------------------------------
# token log probabilities
# ----------------------------------------------------------------------------
from test_gpu_reading import logprobs_check  # noqa: E402


@pytest.mark.parametrize("temperature,up", [(8e37, 1e30), (2e36, 1e30), (1e33, 1.0), (2e-38, 1e-3)])
@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_gradients_at_extreme_temperatures(V, temperature, up):
    # upstream gradients that leave results among float32's normal numbers
    m = Make(V)
    z = m.act(4, V)
    z[1, ::2] = -INF
    z[2, :V // 2] = -INF
    z[3, 1:] = -INF
    print(f"extreme temperatures V={V} {temperature}", flush=True)
    tokens, g = i32([0, 1, V - 1, 0]), [m.f32(4, scale=up), m.f32(4, scale=up), m.f32(4, 5, scale=up)]
    logprobs_check(z, tokens, 5, temperature, *g)
    logprobs_check(z, tokens, 5, temperature, g[0])
    logprobs_check(z, tokens, 5, temperature, gentropy=g[1])
    logprobs_check(z, None, 5, temperature, gtop=g[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [40, 3000, 40000, 140000])
def test_gradients_of_rows_with_holes(V, dtype):
    # each place's gradient against its own terms
    m = Make(V, dtype)
    z = m.act(5, V)
    z[0, 1:] = -INF
    z[1, ::2] = -INF
    z[2, V // 2:] = -INF
    z[3, torch.randperm(V, generator=m.g)[:V - V // 8].cuda()] = -INF
    print(f"holes V={V} {dtype}", flush=True)
    tokens, K = i32([0, 1, V - 1, -1, V // 2]), 20
    logprobs_check(z, tokens, K, 1.0, m.f32(5), m.f32(5), m.f32(5, K))
    logprobs_check(z, tokens, K, 0.7, m.f32(5), m.f32(5))
    logprobs_check(z, None, 0, 1.0, gentropy=m.f32(5))


# ----------------------------------------------------------------------------
# refusals
# ----------------------------------------------------------------------------
def test_positions_without_axes_are_refused():
    m = Make(1)
    x, f = m.act(2, 3, 4, 16), m.f32(8)
    for t, positions in ((x, torch.tensor(3, dtype=torch.int32, device="cuda")), (x[:, 0], m.ints(0, 9, 2)),
                         (x[:, 0], torch.tensor(3, dtype=torch.int32, device="cuda")), (x, m.ints(0, 9, 3))):
        with pytest.raises(ValueError, match="positions"):
            seq.rotary_forward(t, positions, f)
