"""Pins of the sequence operators' oracle: closed forms, torch's own functions, and every gradient
against central differences (float64, on the CPU)."""

import numpy as np
import pytest
import torch

from oracle import sequence as seq


def _differences(f, arrays, names, eps=1e-6):
    """Gradients of the scalar f(**arrays) by central differences."""
    out = {}
    for k in names:
        g = np.zeros_like(arrays[k])
        for i in np.ndindex(*g.shape):
            v = arrays[k][i]
            arrays[k][i] = v + eps
            hi = f(**arrays)
            arrays[k][i] = v - eps
            lo = f(**arrays)
            arrays[k][i] = v
            g[i] = (hi - lo) / (2 * eps)
        out[k] = g
    return out


def _close(got, want):
    # central differences at 1e-6: truncation about 1e-12 of the third derivative, rounding about 1e-10
    assert got.shape == want.shape
    assert np.abs(got - want).max() <= 1e-7 * max(1.0, np.abs(want).max())


@pytest.mark.parametrize("silu", [False, True])
def test_causal_conv_equals_torch(silu):
    rng = np.random.default_rng(1)
    x, w, bias = rng.standard_normal((2, 9, 5)), rng.standard_normal((5, 4)), rng.standard_normal(5)
    y, new = seq.causal_conv(x, w, bias, silu)
    t = torch.from_numpy(x).transpose(1, 2)
    want = torch.nn.functional.conv1d(torch.nn.functional.pad(t, (3, 0)), torch.from_numpy(w)[:, None],
                                      torch.from_numpy(bias), groups=5)
    want = torch.nn.functional.silu(want) if silu else want
    np.testing.assert_allclose(y, want.transpose(1, 2).numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_array_equal(new, x[:, -3:])
    # two calls with the state in between are one call
    a, s = seq.causal_conv(x[:, :2], w, bias, silu)
    b, s = seq.causal_conv(x[:, 2:], w, bias, silu, state=s)
    np.testing.assert_allclose(np.concatenate([a, b], 1), y, rtol=1e-12, atol=1e-12)
    np.testing.assert_array_equal(s, new)


@pytest.mark.parametrize("silu", [False, True])
def test_causal_conv_gradients(silu):
    rng = np.random.default_rng(2)
    v = {"x": rng.standard_normal((3, 6, 2)), "w": rng.standard_normal((2, 3)), "bias": rng.standard_normal(2)}
    state, lengths, gy = rng.standard_normal((3, 2, 2)), [6, 0, 3], rng.standard_normal((3, 6, 2))
    gx, gw, gb = seq.causal_conv_backward(gy, v["x"], v["w"], v["bias"], silu, state, lengths)
    want = _differences(lambda **k: (seq.causal_conv(silu=silu, state=state, lengths=lengths, **k)[0] * gy).sum(), v,
                        ("x", "w", "bias"))
    for got, k in ((gx, "x"), (gw, "w"), (gb, "bias")):
        _close(got, want[k])


def test_scan_closed_forms():
    # one channel, one state, constant step: h[t] = sum_k exp(-k d) d x, a geometric sum
    L, d = 12, 0.3
    one = np.ones((1, L, 1))
    y, h, _ = seq.scan(one, d * one, -np.ones((1, 1)), one[..., None], one[..., None], softplus=False)
    want = d * (1 - np.exp(-d * np.arange(1, L + 1))) / (1 - np.exp(-d))
    np.testing.assert_allclose(y[0, :, 0], want, rtol=1e-12)
    np.testing.assert_allclose(h[0, 0, 0], want[-1], rtol=1e-12)
    # A = 0: the running sum of delta x B; softplus(0) = log 2
    y, _, _ = seq.scan(one, 0 * one, np.zeros((1, 1)), one[..., None], one[..., None])
    np.testing.assert_allclose(y[0, :, 0], np.log(2) * np.arange(1, L + 1), rtol=1e-12)


def _scan_inputs(rng, nb, L, D, N, G):
    return {"x": rng.standard_normal((nb, L, D)), "dt": rng.standard_normal((nb, L, D)),
            "A": -np.exp(rng.standard_normal((D, N))), "B": rng.standard_normal((nb, L, G, N)),
            "C": rng.standard_normal((nb, L, G, N)), "skip": rng.standard_normal(D),
            "gate": rng.standard_normal((nb, L, D)), "dt_bias": rng.standard_normal(D)}


def test_scan_in_two_calls_is_one():
    v = _scan_inputs(np.random.default_rng(3), 2, 9, 4, 3, 2)
    y, h, _ = seq.scan(**v)
    cut = lambda a, b: {k: t[:, a:b] if t.ndim > 2 else t for k, t in v.items()}  # noqa: E731
    y0, h0, _ = seq.scan(**cut(0, 4))
    y1, h1, _ = seq.scan(h0=h0, **cut(4, 9))
    np.testing.assert_allclose(np.concatenate([y0, y1], 1), y, rtol=1e-12)
    np.testing.assert_allclose(h1, h, rtol=1e-12)


@pytest.mark.parametrize("softplus", [False, True])
def test_scan_gradients(softplus):
    rng = np.random.default_rng(4)
    v = _scan_inputs(rng, 3, 5, 4, 2, 2)
    if not softplus:
        v["dt"] = np.abs(v["dt"]) * 0.3
        v["dt_bias"] = np.abs(v["dt_bias"]) * 0.1
    h0, lengths, gy = rng.standard_normal((3, 4, 2)), [5, 0, 3], rng.standard_normal((3, 5, 4))
    got = seq.scan_backward(gy, softplus=softplus, h0=h0, lengths=lengths, **v)
    want = _differences(lambda **k: (seq.scan(softplus=softplus, h0=h0, lengths=lengths, **k)[0] * gy).sum(), v, v)
    for k in v:
        _close(got[k], want[k])


PARTS = [(), ("w_pre",), ("f",), ("f", "w_post"), ("f", "gate", "w_pre"), ("f", "scale", "w_post"),
         ("f", "gate", "scale", "w_post", "w_pre")]


@pytest.mark.parametrize("parts", PARTS[1:])
@pytest.mark.parametrize("act", ["none", "sigmoid", "silu"])
def test_block_norm_gradients(parts, act):
    rng = np.random.default_rng(5)
    R, D = 3, 5
    v = {"x": rng.standard_normal((R, D))}
    v.update({k: rng.standard_normal((R, D) if k in ("f", "gate") else D) for k in parts})
    gout, gn = rng.standard_normal((2, R, D))

    def loss(**k):
        out, n = seq.block_norm(act=act, **k)
        return (out * gout).sum() + (0 if n is None else (n * gn).sum())

    got = seq.block_norm_backward(gout, gn, act=act, **v)
    want = _differences(loss, v, v)
    assert got.keys() == want.keys()
    for k in v:
        _close(got[k], want[k])


def test_block_norm_of_unit_rows():
    x = np.array([[3.0, -3.0, 3.0, -3.0]])
    out, n = seq.block_norm(x, w_pre=np.ones(4), eps=1e-30)
    np.testing.assert_allclose(n, np.sign(x), rtol=1e-12)
    np.testing.assert_array_equal(out, x)


def test_distill_equals_torch():
    rng = np.random.default_rng(6)
    R, V, tau, alpha = 4, 7, 2.5, 0.3
    z, teacher = rng.standard_normal((R, V)), rng.standard_normal((R, V))
    labels = rng.integers(0, V, R)
    loss, _ = seq.distill(z, np.tile(np.arange(V), (R, 1)), teacher, tau, labels, alpha)
    tz, tt = torch.from_numpy(z), torch.from_numpy(teacher)
    kl = torch.nn.functional.kl_div(torch.log_softmax(tz / tau, 1), torch.log_softmax(tt / tau, 1), log_target=True,
                                    reduction="none").sum(1)
    ce = torch.nn.functional.cross_entropy(tz, torch.from_numpy(labels), reduction="none")
    np.testing.assert_allclose(loss, ((1 - alpha) * ce + alpha * tau ** 2 * kl).numpy(), rtol=1e-12)
    # a student equal to the teacher loses nothing to it
    same, gz = seq.distill(teacher, np.tile(np.arange(V), (R, 1)), teacher, tau)
    assert np.abs(same).max() < 1e-12 and np.abs(gz).max() < 1e-12


def test_distill_gradients():
    rng = np.random.default_rng(7)
    R, V, K = 6, 9, 3
    z = {"z": rng.standard_normal((R, V))}
    idx = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    idx[1], idx[2, 0], idx[3, 1] = -1, -1, idx[3, 0]  # no teacher; one entry absent; one place twice
    labels, weight = np.array([0, 3, -1, 5, 8, 1]), np.array([1, 2, 0.5, 1, 0, 1.0])
    teacher, gloss = rng.standard_normal((R, K)), rng.standard_normal(R)
    kw = {"idx": idx, "teacher": teacher, "temperature": 1.7, "labels": labels, "alpha": 0.6, "weight": weight}
    _, gz = seq.distill(gloss=gloss, **z, **kw)
    want = _differences(lambda z: (seq.distill(z, **kw)[0] * gloss).sum(), z, ("z",))
    _close(gz, want["z"])
    assert not gz[4].any()
