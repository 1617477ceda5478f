"""The sequence operators on the GPU against the float64 oracle, at the sizes, masks and strides where
they can go wrong.

Tolerances.  Every sum is formed in float32 and each output rounded once to its type, so a result is
off by at most
  u |ref| (u = 2^-8, 2^-11, 2^-24: the unit roundoff of bfloat16, float16 and float32)
from its rounding, and by float32 errors of what led to it: a few hundred terms at most, each off by
a few units of 2^-24 relative to its own size, exponentials by some 2^-22 after their argument's
rounding, adding up like at most 300 * 2^-24 = 2e-5 of the largest intermediate, which the largest
result of a tensor stands for.  So every element has to lie within
  u |ref| + 4e-5 max|ref| (+ float16's subnormal spacing, 2^-24)
and the relative 2-norm within u + 2e-5.
"""

import numpy as np
import pytest
import torch

from oracle import sequence as oracle
from paper_2106_12736_amd import sequence as seq
from paper_2106_12736_amd._lib import FdcError

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check(got, want, name):
    u = UNIT[got.dtype]
    tiny = 2.0 ** -24 if got.dtype == torch.float16 else 1e-30
    got, want = host(got), np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(inf, np.isinf(got)) and np.array_equal(got[inf], want[inf]), f"{name}: infinities"
    on = np.isfinite(want)
    got, want = got[on], want[on]
    if not want.size:
        return
    off = np.abs(got - want)
    worst = np.abs(want).max()
    assert (off <= u * np.abs(want) + 4e-5 * worst + tiny).all(), f"{name}: off by {off.max():.3e}, largest {worst:.3e}"
    norm = np.linalg.norm(want)
    assert np.linalg.norm(off) <= (u + 2e-5) * norm + tiny * np.sqrt(want.size), f"{name}: {np.linalg.norm(off) / norm:.3e}"


class Make:
    """Seeded inputs on the GPU."""

    def __init__(self, seed, dtype="f32"):
        self.g = torch.Generator().manual_seed(seed)
        self.dtype = DTYPES[dtype]

    def f32(self, *shape, scale=1.0, mean=0.0):
        return (torch.randn(shape, generator=self.g) * scale + mean).cuda()

    def act(self, *shape, scale=1.0):
        return self.f32(*shape, scale=scale).to(self.dtype)


def strided(t, how):
    """The same values in another layout: a slice of wider rows, tokens outside batch, one element off
    alignment."""
    if how == "dense":
        return t
    if how == "slice":
        wide = torch.full(t.shape[:-1] + (t.shape[-1] * 2 + 3,), float("nan"), dtype=t.dtype, device=t.device)
        out = wide[..., 3:3 + t.shape[-1]]
    elif how == "tokens_first":
        out = torch.empty((t.shape[1], t.shape[0]) + t.shape[2:], dtype=t.dtype, device=t.device).transpose(0, 1)
    elif how == "off":
        out = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    return out.copy_(t)


def poison(t, lengths):
    """NaN at the tokens beyond each sequence's length."""
    if lengths is not None:
        for b, n in enumerate(lengths.tolist()):
            t[b, min(max(n, 0), t.shape[1]):] = float("nan")
    return t


# ----------------------------------------------------------------------------
# causal convolution
# ----------------------------------------------------------------------------
def conv_case(B, L, D, n, dtype, silu, bias, state, lengths, layout="dense", seed=0):
    print(f"conv B={B} L={L} D={D} n={n} {dtype} silu={silu} bias={bias} state={state} lengths={lengths} {layout}",
          flush=True)
    m = Make(seed, dtype)
    lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    x, gy = (strided(poison(m.act(B, L, D), lengths), layout) for _ in range(2))
    w, b = m.f32(D, n), m.f32(D) if bias else None
    st = m.act(B, n - 1, D) if state else None
    kw = {"bias": b, "silu": silu, "state": st, "lengths": lengths}
    hk = {"bias": host(b), "silu": silu, "state": host(st), "lengths": None if lengths is None else host(lengths)}
    y, new = seq.causal_conv_forward(x, w, last=True, **kw)
    ry, rnew = oracle.causal_conv(host(x), host(w), **hk)
    check(y, ry, "y")
    assert np.array_equal(host(new), rnew)
    grads = seq.causal_conv_backward(gy, x, w, **kw)
    for got, want, name in zip(grads, oracle.causal_conv_backward(host(gy), host(x), host(w), **hk), ("gx", "gw", "gbias")):
        if got is not None:
            check(got, want, name)
    assert (grads[2] is None) == (b is None)
    return y, new


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_conv_taps(n, dtype):
    conv_case(2, 21, 19, n, dtype, True, True, True, None, seed=n)


@pytest.mark.parametrize("B,L,D", [(1, 1, 1), (1, 1, 8), (3, 2, 7), (1, 3, 64), (2, 9, 130), (1, 100, 5),
                                   (2, 70, 520), (5, 33, 12)])
def test_conv_sizes(B, L, D):
    conv_case(B, L, D, 4, "bf16", True, True, False, None, seed=L)
    conv_case(B, L, D, 3, "f32", False, False, True, None, seed=D)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 40], [2, 17, 39], [40, -3, 99]])
@pytest.mark.parametrize("state", [False, True])
def test_conv_lengths(lengths, state):
    conv_case(3, 40, 33, 4, "bf16", True, True, state, lengths)
    conv_case(3, 40, 33, 8, "f32", False, True, state, lengths)


@pytest.mark.parametrize("layout", ["slice", "tokens_first", "off"])
def test_conv_layouts(layout):
    conv_case(3, 25, 24, 4, "bf16", True, True, True, [25, 7, 0], layout)
    conv_case(2, 25, 23, 3, "f32", False, True, False, None, layout)


def test_conv_long_run_with_many_sums():
    # enough tokens and channels that a thread walks more than the shortest run
    B, L, D, n = 2, 4096, 2048, 4
    print(f"conv long B={B} L={L} D={D}", flush=True)
    m = Make(9, "bf16")
    x, gy, w, b = m.act(B, L, D), m.act(B, L, D), m.f32(D, n), m.f32(D)
    y, _ = seq.causal_conv_forward(x, w, bias=b, silu=True)
    gx, gw, gb = seq.causal_conv_backward(gy, x, w, bias=b, silu=True)
    some = [0, 1, 777, 2047]
    ref = oracle.causal_conv(host(x[:, :, some]), host(w[some]), host(b[some]), True)[0]
    check(y[:, :, some], ref, "y")
    rx, rw, rb = oracle.causal_conv_backward(host(gy[:, :, some]), host(x[:, :, some]), host(w[some]), host(b[some]), True)
    check(gx[:, :, some], rx, "gx")
    check(gw[some], rw, "gw")
    check(gb[some], rb, "gbias")


def test_conv_steps_equal_one_call():
    m = Make(3, "bf16")
    x, w, b = m.act(3, 11, 40), m.f32(40, 4), m.f32(40)
    y, new = seq.causal_conv_forward(x, w, bias=b, silu=True, last=True)
    state = torch.zeros(3, 3, 40, dtype=torch.bfloat16, device="cuda")
    for t in range(11):
        yt, same = seq.causal_conv_step(x[:, t], w, state, bias=b, silu=True)
        assert same is state and torch.equal(yt, y[:, t])
    assert torch.equal(state, new)
    # the state of an earlier call, updated in place by a longer one
    state = m.act(3, 3, 40)
    want = oracle.causal_conv(host(x), host(w), host(b), True, host(state), [11, 1, 0])[1]
    a = seq._conv_args(x, w, b, True, state, torch.tensor([11, 1, 0], dtype=torch.int32).cuda(), y, state)
    seq.call("fdc_causal_conv_forward", a, seq._stream())
    assert np.array_equal(host(state), want)


# ----------------------------------------------------------------------------
# selective scan
# ----------------------------------------------------------------------------
def scan_inputs(m, B, L, D, N, G, gate, skip, dt_bias, softplus, lengths, layout):
    lead = (B,) if L is None else (B, L)
    lay = lambda t: strided(poison(t, lengths) if L else t, layout)  # noqa: E731
    v = {"x": lay(m.act(*lead, D)), "dt": lay(m.act(*lead, D, scale=0.7) if softplus else m.act(*lead, D, scale=0.2).abs()),
         "A": -torch.exp(m.f32(D, N, scale=0.7)), "B": poison(m.act(*lead, G, N), lengths),
         "C": poison(m.act(*lead, G, N), lengths), "skip": m.f32(D) if skip else None,
         "gate": lay(m.act(*lead, D)) if gate else None, "dt_bias": m.f32(D, mean=-1.0) if dt_bias else None}
    if not softplus and dt_bias:
        v["dt_bias"] = v["dt_bias"].abs() * 0.1
    return v


def scan_case(B, L, D, N, G=1, dtype="f32", gate=True, skip=True, dt_bias=True, softplus=True, state=False,
              lengths=None, layout="dense", seed=0, channels=None):
    print(f"scan B={B} L={L} D={D} N={N} G={G} {dtype} gate={gate} skip={skip} dt_bias={dt_bias} softplus={softplus} "
          f"state={state} lengths={lengths} {layout}", flush=True)
    m = Make(seed, dtype)
    lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    v = scan_inputs(m, B, L, D, N, G, gate, skip, dt_bias, softplus, lengths, layout)
    h0 = m.f32(B, D, N) if state else None
    gy = strided(poison(m.act(B, L, D), lengths), layout)
    y, h, saved = seq.scan_forward(**v, softplus=softplus, h0=h0, lengths=lengths, last=True, save=True)
    hv = {k: host(t) for k, t in v.items()}
    hk = {"softplus": softplus, "h0": host(h0), "lengths": None if lengths is None else host(lengths)}
    ry, rh, _ = oracle.scan(**hv, **hk)
    check(y, ry, "y")
    check(h, rh, "h_last")
    g = seq.scan_backward(gy, saved, **v, softplus=softplus, lengths=lengths)
    want = oracle.scan_backward(host(gy), **hv, **hk)
    for k in v:
        got = getattr(g, k)
        assert (got is None) == (v[k] is None)
        if got is not None:
            check(got, want[k], "g" + k)


@pytest.mark.parametrize("N", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 60, 64])
def test_scan_states(N):
    scan_case(2, 21, 11, N, dtype="bf16", seed=N)
    scan_case(1, 35, 70, N, dtype="f32", state=True, seed=N)


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 31, 32, 33, 65])
def test_scan_lengths_of_one_call(L):
    scan_case(2, L, 20, 16, dtype="f16", seed=L)
    scan_case(1, L, 5, 8, dtype="f32", state=True, seed=L)


@pytest.mark.parametrize("D,G", [(1, 1), (2, 2), (63, 1), (64, 1), (65, 1), (66, 2), (130, 2), (12, 4), (260, 4)])
def test_scan_groups(D, G):
    scan_case(2, 19, D, 16, G, dtype="bf16", seed=D)
    scan_case(2, 19, D, 10, G, dtype="f32", seed=D)


@pytest.mark.parametrize("gate,skip,dt_bias,softplus", [(False, False, False, False), (True, False, False, True),
                                                        (False, True, False, True), (False, False, True, False)])
def test_scan_parts(gate, skip, dt_bias, softplus):
    scan_case(2, 37, 30, 16, 2, "f32", gate, skip, dt_bias, softplus, state=True)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 75], [16, 17, 33], [75, -2, 90], [15, 32, 74]])
@pytest.mark.parametrize("state", [False, True])
def test_scan_ragged(lengths, state):
    scan_case(3, 75, 40, 16, 2, "bf16", state=state, lengths=lengths)
    scan_case(3, 75, 21, 5, 1, "f32", state=state, lengths=lengths)


@pytest.mark.parametrize("layout", ["slice", "tokens_first", "off"])
def test_scan_layouts(layout):
    scan_case(3, 40, 24, 16, 1, "bf16", lengths=[40, 7, 0], layout=layout)
    scan_case(2, 40, 23, 12, 1, "f32", layout=layout)


@pytest.mark.parametrize("L,D,N,G", [(1000, 8, 16, 1), (513, 20, 40, 2), (640, 3, 4, 1), (2049, 4, 64, 1)])
@pytest.mark.parametrize("lengths", [None, "short"])
def test_scan_long(L, D, N, G, lengths):
    # few channels, many tokens: the work is cut along the tokens
    scan_case(2, L, D, N, G, "f32", state=True, lengths=lengths and [L - 3, L // 3], seed=L)


def test_scan_decays_from_none_to_all():
    # steps from (almost) nothing, where softplus has to keep small values, to ones that wipe the state out
    m = Make(5)
    B, L, D, N = 1, 48, 32, 16
    v = scan_inputs(m, B, L, D, N, 1, False, False, False, True, None, "dense")
    v["dt"] = torch.linspace(-30, 60, D).cuda().expand(B, L, D).contiguous()
    y, h, saved = seq.scan_forward(**v, last=True, save=True)
    hv = {k: host(t) for k, t in v.items()}
    ry, rh, _ = oracle.scan(**hv)
    gy = m.act(B, L, D)
    g, want = seq.scan_backward(gy, saved, **v), oracle.scan_backward(host(gy), **hv)
    for d in range(D):  # channel by channel: each has its own magnitude
        check(y[..., d], ry[..., d], f"y {d}")
        check(h[:, d], rh[:, d], f"h {d}")
        check(g.dt[..., d], want["dt"][..., d], f"gdt {d}")
        check(g.A[d], want["A"][d], f"gA {d}")


@pytest.mark.parametrize("N,G,dtype", [(16, 1, "bf16"), (16, 2, "f16"), (5, 1, "f32"), (64, 4, "bf16"), (30, 1, "f32")])
def test_scan_step(N, G, dtype):
    print(f"scan step N={N} G={G} {dtype}", flush=True)
    m = Make(N, dtype)
    B, D, L = 3, 36, 5
    v = scan_inputs(m, B, L, D, N, G, True, True, True, True, None, "dense")
    h = m.f32(B, D, N)
    ry, rh, states = oracle.scan(**{k: host(t) for k, t in v.items()}, h0=host(h))
    token = lambda t: {k: a[:, t] if k in ("x", "dt", "B", "C", "gate") else a for k, a in v.items()}  # noqa: E731
    y, new = seq.scan_step(**token(0), h=h, h_new=torch.empty_like(h))
    check(y, ry[:, 0], "y")
    check(new, states[:, 1], "h")
    for t in range(L):
        y, same = seq.scan_step(**token(t), h=h)
        assert same is h
        check(y, ry[:, t], f"y {t}")
    check(h, rh, "h")


def test_scan_repeats_bit_for_bit():
    m = Make(8, "bf16")
    v = scan_inputs(m, 2, 700, 96, 16, 1, True, True, True, True, None, "dense")
    gy = m.act(2, 700, 96)
    runs = []
    for _ in range(3):
        y, h, saved = seq.scan_forward(**v, last=True, save=True)
        runs.append([y, h, *(t for t in seq.scan_backward(gy, saved, **v))])
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


# ----------------------------------------------------------------------------
# block norm
# ----------------------------------------------------------------------------
def norm_case(R, D, parts=("f", "gate", "scale", "w_post", "w_pre"), act="silu", dtype="f32", layout="dense", seed=0,
              gout=True, gn=True):
    print(f"norm R={R} D={D} {parts} {act} {dtype} {layout}", flush=True)
    m = Make(seed, dtype)
    lay = lambda t: strided(t, layout)  # noqa: E731
    v = {"x": lay(m.act(R, D))}
    v.update({k: lay(m.act(R, D)) if k in ("f", "gate") else m.f32(D) for k in parts})
    hv = {k: host(t) for k, t in v.items()}
    out, n, stats = seq.block_norm_forward(**v, act=act)
    rout, rn = oracle.block_norm(**hv, act=act)
    check(out, rout, "out")
    assert (n is None) == (rn is None)
    if n is not None:
        check(n, rn, "n")
    go = lay(m.act(R, D)) if gout or n is None else None
    gnv = lay(m.act(R, D)) if gn and n is not None else None
    g = seq.block_norm_backward(go, gnv, stats, **v, act=act)
    want = oracle.block_norm_backward(host(go), host(gnv), **hv, act=act)
    for k in g._fields:
        got = getattr(g, k)
        assert (got is None) == (k not in want), k
        if got is not None:
            check(got, want[k], "g" + k)


@pytest.mark.parametrize("D", [1, 2, 3, 31, 64, 255, 256, 257, 512, 513, 1000, 1025, 2048, 2049, 4095, 4097, 8191, 8192])
def test_norm_widths(D):
    norm_case(3, D, dtype="bf16", seed=D)
    norm_case(5, D, dtype="f32", act="sigmoid", seed=D)


@pytest.mark.parametrize("R", [1, 2, 3, 4, 5, 63, 257, 1500])
def test_norm_rows(R):
    norm_case(R, 72, dtype="f16", seed=R)
    norm_case(R, 300, dtype="f32", act="none", seed=R)


@pytest.mark.parametrize("parts", [("w_pre",), ("f",), ("f", "w_post"), ("f", "gate", "w_pre"), ("f", "scale", "w_pre"),
                                   ("f", "scale", "w_post"), ("f", "gate", "scale", "w_post")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_parts(parts, dtype):
    norm_case(9, 130, parts, "sigmoid", dtype)


@pytest.mark.parametrize("layout", ["slice", "off"])
def test_norm_layouts(layout):
    norm_case(7, 120, dtype="bf16", layout=layout)
    norm_case(7, 121, dtype="f32", layout=layout)


def test_norm_one_gradient_alone():
    norm_case(6, 200, gout=False)
    norm_case(6, 200, gn=False)


def test_norm_rows_of_zeros_and_large_values():
    m = Make(1)
    x, f = m.act(4, 96), m.act(4, 96)
    x[0], f[0], x[1] = 0, 0, 1e15
    f[2] = 1e-15
    w = torch.ones(96, device="cuda")
    out, n, stats = seq.block_norm_forward(x, f, w_post=w, w_pre=w)
    rout, rn = oracle.block_norm(host(x), host(f), w_post=host(w), w_pre=host(w))
    g = seq.block_norm_backward(x, f, stats, x, f, w_post=w, w_pre=w)
    want = oracle.block_norm_backward(host(x), host(f), host(x), host(f), w_post=host(w), w_pre=host(w))
    for r in range(4):
        check(out[r], rout[r], f"out {r}")
        check(n[r], rn[r], f"n {r}")
        if r != 1:  # its gradient is the difference of two numbers of 1e15
            check(g.x[r], want["x"][r], f"gx {r}")
            check(g.f[r], want["f"][r], f"gf {r}")


def test_norm_expanded_gate():
    m = Make(2, "bf16")
    x, f, one = m.act(6, 64), m.act(6, 64), m.act(1, 64)
    a = seq.block_norm_forward(x, f, one.expand(6, 64))[0]
    assert torch.equal(a, seq.block_norm_forward(x, f, one.expand(6, 64).contiguous())[0])


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------
def distill_case(R, V, K, dtype="f32", tau=2.0, alpha=0.7, labels=True, weight=True, holes=True, layout="dense", seed=0,
                 change=None):
    print(f"distill R={R} V={V} K={K} {dtype} tau={tau} alpha={alpha} {layout}", flush=True)
    m = Make(seed, dtype)
    z = strided(m.act(R, V, scale=3.0), layout)
    idx = torch.stack([torch.randperm(V, generator=m.g)[:K] for _ in range(R)]).int().cuda()
    teacher = m.act(R, K, scale=2.0)
    lab = torch.randint(0, V, (R,), generator=m.g).int().cuda() if labels else None
    w = m.f32(R).abs() if weight else None
    if holes:
        idx[0] = -1
        idx[R // 2, K // 2:] = -1
        if labels:
            lab[R - 1] = -5
        if weight:
            w[R // 3] = 0
            z[R // 3] = float("nan")
    v = {"z": z, "idx": idx, "teacher": teacher, "labels": lab, "weight": w}
    if change:
        change(v)
    gloss = m.f32(R)
    kw = {**v, "temperature": tau, "alpha": alpha}
    hv = {k: None if t is None else t.cpu().numpy() if t.dtype == torch.int32 else host(t) for k, t in v.items()}
    rloss, rgz = oracle.distill(**hv, temperature=tau, alpha=alpha, gloss=host(gloss))
    loss, stats = seq.distill_forward(**kw)
    check(loss, rloss, "loss")
    gz = seq.distill_backward(gloss, stats, **kw)
    both, gz2 = seq.distill_forward_backward(gloss, **kw)
    check(both, rloss, "loss in one call")
    for r in range(R):
        check(gz[r], rgz[r], f"gz {r}")
        check(gz2[r], rgz[r], f"gz in one call {r}")
    inplace = z.clone()
    seq.distill_backward(gloss, stats, **{**kw, "z": inplace}, gz=inplace)
    assert torch.equal(inplace.nan_to_num(7.0), gz.nan_to_num(7.0))
    return loss, gz


@pytest.mark.parametrize("V,K", [(1, 1), (2, 2), (7, 3), (64, 64), (255, 5), (1000, 1), (2047, 100), (4097, 64),
                                 (33000, 1024)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_distill_sizes(V, K, dtype):
    distill_case(5, V, K, dtype, seed=V)


@pytest.mark.parametrize("tau,alpha,labels,weight", [(1.0, 1.0, False, False), (1.0, 0.5, True, False), (0.3, 1.0, True, True),
                                                     (8.0, 0.0, True, True), (2.0, 0.25, True, True)])
def test_distill_terms(tau, alpha, labels, weight):
    distill_case(6, 501, 17, "f32", tau, alpha, labels, weight)
    distill_case(6, 504, 17, "bf16", tau, alpha, labels, weight)


@pytest.mark.parametrize("layout", ["slice", "off"])
def test_distill_layouts(layout):
    distill_case(4, 777, 9, "bf16", layout=layout)
    distill_case(4, 776, 9, "f32", layout=layout)


@pytest.mark.parametrize("R,V", [(1, 130000), (2, 50021), (700, 3001), (3000, 40)])
def test_distill_shapes(R, V):
    distill_case(R, V, 12, "bf16" if R < 1000 else "f32", seed=R)


@pytest.mark.parametrize("R,V,dtype", [(260, 60, "f32"), (260, 2000, "f16"), (260, 7001, "bf16"), (260, 16384, "bf16"),
                                       (770, 20001, "bf16"), (770, 20001, "f16"), (770, 12000, "f32"), (770, 20001, "f32")])
def test_distill_rows_in_registers(R, V, dtype):
    # a workgroup a row, in each of its widths
    distill_case(R, V, 20, dtype, seed=R)


def test_distill_masked_and_odd_values():
    lowest = {"f32": torch.finfo(torch.float32).min, "bf16": torch.finfo(torch.bfloat16).min, "f16": -65504.0}

    def change(v):
        z, idx, t = v["z"], v["idx"], v["teacher"]
        at = idx[1].long()
        free = [c for c in range(z.shape[1]) if c not in set(at.tolist()) | {int(v["labels"][1])}]
        z[1, free[:50]] = float("-inf")           # a vocabulary masked with -inf
        z[1, free[50:90]] = lowest[name]          # and with the type's lowest value
        t[2, :3] = float("-inf")                  # teacher entries of no probability
        idx[3, 1] = idx[3, 0]                     # one place given twice
        t[4] = float("-inf")                      # a teacher that says nothing
        idx[5, 2] = z.shape[1]                    # an index past the vocabulary
        v["labels"][6] = z.shape[1]               # a label past it
        z[7] = float("-inf")                      # a row of nothing at all

    for name in lowest:
        distill_case(8, 301, 8, name, tau=1.5, weight=False, holes=False, change=change)


def test_distill_repeats_bit_for_bit():
    m = Make(4, "bf16")
    z, teacher = m.act(40, 9000, scale=3.0), m.act(40, 30)
    idx = torch.stack([torch.randperm(9000, generator=m.g)[:30] for _ in range(40)]).int().cuda()
    gloss = m.f32(40)
    a, b = (seq.distill_forward_backward(gloss, z, idx, teacher) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ----------------------------------------------------------------------------
# streams, graphs, refusals
# ----------------------------------------------------------------------------
def _everything(v):
    y, st = seq.causal_conv_forward(v["x"], v["w"], bias=v["skip"], silu=True, last=True)
    gx, gw, gb = seq.causal_conv_backward(v["gate"], v["x"], v["w"], bias=v["skip"], silu=True)
    s = {k: v[k] for k in ("x", "dt", "A", "B", "C", "skip", "gate", "dt_bias")}
    ys, h, saved = seq.scan_forward(**s, last=True, save=True)
    g = seq.scan_backward(y, saved, **s)
    rows = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    out, n, stats = seq.block_norm_forward(rows(v["x"]), rows(ys), rows(v["gate"]), v["skip"], v["skip"], v["skip"])
    gn = seq.block_norm_backward(out, n, stats, rows(v["x"]), rows(ys), rows(v["gate"]), v["skip"], v["skip"], v["skip"])
    loss, gz = seq.distill_forward_backward(v["gloss"], n, v["idx"], v["teacher"])
    return [y, st, gx, gw, gb, ys, h, *g, out, n, *gn, loss, gz]


def _all_inputs():
    m = Make(11, "bf16")
    B, L, D = 2, 600, 48
    v = scan_inputs(m, B, L, D, 16, 1, True, True, True, True, None, "dense")
    v.update(w=m.f32(D, 4), gloss=m.f32(B * L), teacher=m.act(B * L, 5),
             idx=torch.stack([torch.randperm(D, generator=m.g)[:5] for _ in range(B * L)]).int().cuda())
    return v


def test_other_streams():
    v = _all_inputs()
    want = _everything(v)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(_everything(v))
    for s, g in zip(streams, got):
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, g))


def test_captured_in_a_graph():
    v = _all_inputs()
    want = [t.clone() for t in _everything(v)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _everything(v)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _everything(v)
    x = v["x"].clone()
    for k in range(3):
        v["x"].copy_(x if k != 1 else x * 0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = _everything(v)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), k
        if k != 1:
            assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_refusals():
    m = Make(1, "bf16")
    x, w = m.act(2, 6, 8), m.f32(8, 4)
    bad = [
        lambda: seq.causal_conv_forward(x.double(), w),
        lambda: seq.causal_conv_forward(x.cpu(), w),
        lambda: seq.causal_conv_forward(x, w.bfloat16()),
        lambda: seq.causal_conv_forward(x, m.f32(7, 4)),
        lambda: seq.causal_conv_forward(x.transpose(1, 2), m.f32(6, 4)),
        lambda: seq.causal_conv_forward(x, w, state=m.act(2, 4, 8)),
        lambda: seq.causal_conv_forward(x, w, lengths=torch.zeros(2, device="cuda")),
        lambda: seq.causal_conv_backward(x[:, :5], x, w),
        lambda: seq.scan_forward(x, x, m.f32(8, 4), m.act(2, 6, 1, 4), m.act(2, 6, 2, 4)),
        lambda: seq.scan_forward(x, x.float(), m.f32(8, 4), m.act(2, 6, 1, 4), m.act(2, 6, 1, 4)),
        lambda: seq.scan_step(x[:, 0], x[:, 0], m.f32(8, 4), m.act(2, 1, 4), m.act(2, 1, 4), m.f32(2, 8, 5)),
        lambda: seq.block_norm_forward(x, x),
        lambda: seq.block_norm_forward(x[0], x[0], act="tanh"),
        lambda: seq.block_norm_forward(x[0], x[0], scale=m.f32(7)),
        lambda: seq.distill_forward(x[0], torch.zeros(6, 2, device="cuda").long(), m.act(6, 2)),
        lambda: seq.distill_forward(x[0], torch.zeros(6, 2, device="cuda").int(), m.act(6, 3)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("accepted", i)
    refused = [
        lambda: seq.causal_conv_forward(x, m.f32(8, 9)),
        lambda: seq.scan_forward(x, x, m.f32(8, 65), m.act(2, 6, 1, 65), m.act(2, 6, 1, 65)),
        lambda: seq.scan_forward(x, x, m.f32(8, 4), m.act(2, 6, 3, 4), m.act(2, 6, 3, 4)),
        lambda: seq.block_norm_forward(m.act(2, 8193)),
        lambda: seq.block_norm_forward(x[0], w_pre=m.f32(8), eps=0.0),
        lambda: seq.block_norm_forward(x[0], scale=m.f32(8), w_pre=m.f32(8)),
        lambda: seq.distill_forward(x[0], torch.zeros(6, 2, device="cuda").int(), m.act(6, 2), temperature=0.0),
        lambda: seq.distill_forward(x[0], torch.zeros(6, 2, device="cuda").int(), m.act(6, 2), alpha=1.5),
    ]
    for i, f in enumerate(refused):
        with pytest.raises(FdcError):
            f()
            print("accepted", i)
