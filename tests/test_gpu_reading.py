"""The operators that read an image's tokens and score answers (rotary positions, cross attention, token log
probabilities) on the GPU against the float64 oracle, at the sizes, masks, strides and values where they can go wrong.

Tolerances.  u is half a step of a type (2^-24, 2^-8, 2^-11).  Every output is rounded once, u |ref|.
  rotary     cosine and sine are off by at most 4 units of 2^-24, two products and their sum by one each: at most
             16 * 2^-24 = 1e-6 of the head's largest channel.
  attention  16-bit types round each factor p (or gradient of a score) of a sum once more, u of the sum of the terms'
             absolute values, which `bounds` forms; float32 errors (products over up to 128 channels, exponents of up to
             some 30, sums) add up like at most 300 * 2^-24 = 2e-5 of the same sums, doubled for what leads to a gradient
             of a score.  bfloat16's delta is formed of y to 16 bits: 2^-17 of |gy| |y|, within the same 4e-5.  That y has
             weights w_j = p_j (1 + e_j) / sum p (1 + e), |e_j| <= u, so that with gp = gy v^T delta is off by
             sum (w_j - p_j) (gp_j - delta) <= u sum p_j |gp_j - delta| (1 + u) / (1 - u), and a score's gradient by p times that.
             float16: its subnormal spacing 2^-24, too.
  logprobs   sums of exponentials to some 100 * 2^-24 relative, differences to 2^-23: 1e-5 (1 + |ref|).  The
             gradient's terms likewise, 4e-5 of their absolute values; an exponential below 2^-126, float32's least
             normal number, is 0, which is off by less than 2^-126 times what it is multiplied with.
"""

import numpy as np
import pytest
import torch

from oracle import reading as oracle
from paper_2106_12736_amd import sequence as seq
from paper_2106_12736_amd._lib import FdcError

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def within(got, want, tol, name):
    """tol: what an element may be off beyond its own rounding."""
    u, tiny = UNIT[got.dtype], 2.0 ** -24 if got.dtype == torch.float16 else 1e-37
    got = host(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{name}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and not np.isinf(got[~inf]).any(), f"{name}: infinities"
    on = np.isfinite(want)
    off = np.abs(np.where(on, got, 0) - np.where(on, want, 0))
    most = u * np.abs(np.where(on, want, 0)) + tol + tiny
    bad = on & ~(off <= most)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size}, off by {off[bad].max():.3e} where {most[bad].min():.3e} is allowed"


class Make:
    """Seeded inputs on the GPU."""

    def __init__(self, seed, dtype="f32"):
        self.g = torch.Generator().manual_seed(seed)
        self.dtype = DTYPES[dtype]

    def f32(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g) * scale).cuda()

    def act(self, *shape, scale=1.0):
        return self.f32(*shape, scale=scale).to(self.dtype)

    def ints(self, low, high, *shape):
        return torch.randint(low, high, shape, generator=self.g, dtype=torch.int32).cuda()


def i32(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32).cuda()


def laid(t, how):
    """The same values [B, L, H, D] in another layout."""
    B, L, H, D = t.shape
    nan = lambda *s: torch.full(s, float("nan"), dtype=t.dtype, device=t.device)  # noqa: E731
    if how == "dense":
        return t
    if how == "heads_first":
        out = nan(B, H, L, D).transpose(1, 2)
    elif how == "tokens_first":
        out = nan(L, B, H, D).transpose(0, 1)
    elif how == "slice":
        out = nan(B, L, 3 * H * D + 5)[..., H * D + 1:2 * H * D + 1].unflatten(-1, (H, D))
    elif how == "wide_heads":
        out = nan(B, L, H, D + 3)[..., 1:D + 1]
    elif how == "off":
        out = nan(t.numel() + 1)[1:].view(t.shape)
    return out.copy_(t)


LAYOUTS = ["heads_first", "tokens_first", "slice", "wide_heads", "off"]


# ----------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------
def rotary_case(B, L, H, D, sections, dtype="f32", interleaved=False, lengths=None, far=1000, shared=False, layout="dense",
                seed=0):
    print(f"rotary B={B} L={L} H={H} D={D} {sections} {dtype} interleaved={interleaved} lengths={lengths} far={far} {layout}",
          flush=True)
    m = Make(seed, dtype)
    x, P = m.act(B, L, H, D), sum(sections)
    for b, n in enumerate(lengths or []):
        x[b, min(max(n, 0), L):] = float("nan")
    x = laid(x, layout)
    pos = m.ints(-far, far, *((L,) if shared else (B, L)), len(sections))
    freqs = torch.exp(-m.f32(P).abs() * 3)
    kw = dict(sections=sections, interleaved=interleaved, lengths=i32(lengths))
    hk = dict(sections=sections, interleaved=interleaved, lengths=lengths)
    largest = np.nan_to_num(np.abs(host(x))).max() * 1e-6
    y = seq.rotary_forward(x, pos, freqs, **kw)
    within(y, oracle.rotary(host(x), pos.cpu().numpy(), host(freqs), **hk), largest, "y")
    gx = seq.rotary_backward(x, pos, freqs, **kw)
    within(gx, oracle.rotary(host(x), pos.cpu().numpy(), host(freqs), inverse=True, **hk), largest, "gx")
    over = laid(x.clone(), layout)
    assert seq.rotary_forward(over, pos, freqs, y=over, **kw) is over and torch.equal(over, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,sections", [(2, (1,)), (8, (4,)), (9, (1, 2)), (16, (3, 4, 1)), (17, (8,)), (33, (2, 1, 5, 8)),
                                        (64, (32,)), (90, (17, 16)), (128, (22, 21, 21)), (100, (3, 2)), (256, (128,))])
def test_rotary_pairs(D, sections, interleaved, dtype):
    rotary_case(2, 5, 3, D, sections, dtype, interleaved, seed=D)


@pytest.mark.parametrize("B,L,H", [(1, 1, 1), (1, 1, 32), (3, 1, 7), (2, 257, 1), (5, 3, 33), (1, 1030, 4)])
def test_rotary_sizes(B, L, H):
    rotary_case(B, L, H, 40, (10, 5), "bf16", seed=L)
    rotary_case(B, L, H, 24, (12,), "f32", True, seed=H)


def test_rotary_many_heads_a_thread():
    rotary_case(4, 2049, 5, 64, (16, 16), "bf16", seed=3)


@pytest.mark.parametrize("far", [1 << 20, 1 << 30])
def test_rotary_far_positions(far):
    rotary_case(2, 30, 2, 32, (8, 8), "f32", far=far)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 40], [40, -3, 99]])
def test_rotary_lengths(lengths):
    rotary_case(3, 40, 3, 22, (4, 4), "bf16", lengths=lengths)
    rotary_case(3, 40, 2, 20, (10,), "f32", True, lengths=lengths)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotary_layouts(layout):
    rotary_case(3, 12, 4, 24, (6, 6), "bf16", layout=layout)
    rotary_case(2, 12, 3, 23, (5,), "f32", True, [12, 5], layout=layout)


def test_rotary_shared_positions_and_one_token():
    rotary_case(3, 9, 2, 16, (4, 4), "f32", shared=True)
    m = Make(8, "bf16")
    x, pos, f = m.act(5, 6, 24), m.ints(0, 50, 5, 3), m.f32(12).abs()
    y = seq.rotary_forward(x, pos, f, sections=(4, 4, 4))
    assert torch.equal(y, seq.rotary_forward(x[:, None], pos[:, None], f, sections=(4, 4, 4))[:, 0])
    # a broadcast input (one row for every token) has a dense output
    wide = x[:, None].expand(5, 7, 6, 24)
    y = seq.rotary_forward(wide, pos[:, None].expand(5, 7, 3), f, sections=(4, 4, 4))
    assert torch.equal(y[:, 0], y[:, 6])


# ----------------------------------------------------------------------------
# cross attention
# ----------------------------------------------------------------------------
def bounds(gy, q, k, v, y, scale, q_lengths, lengths, mask):
    """Sums of absolute values of the terms of y, gq, gk and gv: with a score's gradient as it is, and as its parts."""
    B, Lq, H, D = q.shape
    G = k.shape[2]
    out = [np.zeros(x.shape) for x in (q, q, k, v)]
    parts = [np.zeros(x.shape) for x in (q, k)]
    for b, n in enumerate(oracle._count(q_lengths, B, Lq)):
        at = oracle._keys(b, k.shape[1], lengths, mask)
        if not len(at) or not n:
            continue
        for h in range(H):
            g = h // (H // G)
            p, _ = oracle._softmax_rows(q[b, :n, h] @ k[b, at, g].T * scale)
            ag, av, aq, ak = (np.abs(x) for x in (gy[b, :n, h], v[b, at, g], q[b, :n, h], k[b, at, g]))
            out[0][b, :n, h] = p @ av
            out[3][b, at, g] += p.T @ ag
            gp = gy[b, :n, h] @ v[b, at, g].T
            gs = np.abs(p * (gp - (p * gp).sum(1, keepdims=True))) * scale
            gs = gs + p * gs.sum(1, keepdims=True) * 1.01  # its rounding, and delta's
            part = p * (ag @ av.T + (ag * np.abs(y[b, :n, h])).sum(1, keepdims=True)) * scale
            out[1][b, :n, h], parts[0][b, :n, h] = gs @ ak, part @ ak
            out[2][b, at, g] += gs.T @ aq
            parts[1][b, at, g] += part.T @ aq
    return out, parts


def attention_case(B, Lq, Lk, H, G, D, dtype="f32", q_lengths=None, lengths=None, mask=None, layout="dense", scale=None,
                   spread=1.0, up=1.0, seed=0):
    print(f"attention B={B} Lq={Lq} Lk={Lk} H={H} G={G} D={D} {dtype} q_lengths={q_lengths} lengths={lengths} "
          f"mask={mask} {layout} spread={spread} up={up}", flush=True)
    m = Make(seed, dtype)
    q, k, v, gy = m.act(B, Lq, H, D, scale=spread), m.act(B, Lk, G, D), m.act(B, Lk, G, D), m.act(B, Lq, H, D, scale=up)
    if isinstance(mask, float):
        mask = (m.f32(B, Lk).cpu() < mask).cuda()
    elif mask is not None:
        mask = torch.tensor(mask).cuda()
    hm = None if mask is None else mask.cpu().numpy()
    for b in range(B):
        hidden = np.ones(Lk, dtype=bool)
        hidden[oracle._keys(b, Lk, lengths, hm)] = False
        hidden = torch.from_numpy(hidden).cuda()
        k[b, hidden], v[b, hidden] = float("nan"), float("inf")
        if q_lengths is not None:
            n = min(max(q_lengths[b], 0), Lq)
            q[b, n:], gy[b, n:] = float("nan"), float("inf")
    q, k, v, gy = (laid(t, layout) for t in (q, k, v, gy))
    kw = dict(scale=scale, q_lengths=i32(q_lengths), lengths=i32(lengths), mask=mask)
    hk = dict(q_lengths=q_lengths, lengths=lengths, mask=hm)
    y, saved = seq.cross_attention_forward(q, k, v, save=True, **kw)
    hq, hkk, hv, hg = host(q), host(k), host(v), host(gy)
    ry, rlse = oracle.cross_attention(hq, hkk, hv, scale, **hk)
    (ay, aq, ak, av), (pq, pk) = bounds(hg, hq, hkk, hv, ry, D ** -0.5 if scale is None else scale, **hk)
    f, u = 2e-5, UNIT[y.dtype] if dtype != "f32" else 0.0
    within(y, ry, (u + f) * ay, "y")
    within(saved[:B * H * Lq].view(B, H, Lq), rlse, f * (1 + np.abs(np.where(np.isinf(rlse), 0, rlse))), "lse")
    again, none = seq.cross_attention_forward(q, k, v, **kw)
    assert none is None and torch.equal(again, y)
    g = seq.cross_attention_backward(gy, y, saved, q, k, v, **kw)
    want = oracle.cross_attention_backward(hg, hq, hkk, hv, scale, **hk)
    for got, ref, tol, name in zip(g, want, (u * aq + 2 * f * pq, u * ak + 2 * f * pk, (u + f) * av), ("gq", "gk", "gv")):
        within(got, ref, tol, name)
    return y, g


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [1, 2, 7, 8, 16, 31, 32, 33, 40, 64, 65, 80, 96, 97, 100, 120, 127, 128])
def test_attention_widths(D, dtype):
    attention_case(2, 9, 70, 2, 1, D, dtype, seed=D)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [3, 5, 9, 13, 30, 47, 63, 73, 83, 94, 103, 126])
def test_attention_widths_between_pieces(D, dtype):
    # several tiles of rows and keys, and few rows, of widths that are not a number of 16-byte pieces
    attention_case(2, 150, 140, 4, 2, D, dtype, q_lengths=[150, 33], lengths=[77, 140], seed=D)
    attention_case(2, 1, 333, 4, 2, D, dtype, lengths=[333, 40], seed=D)


@pytest.mark.parametrize("Lk", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200])
def test_attention_numbers_of_keys(Lk):
    attention_case(2, 5, Lk, 2, 2, 48, "bf16", seed=Lk)
    attention_case(1, 40, Lk, 3, 1, 24, "f32", seed=Lk)
    attention_case(1, 40, Lk, 2, 1, 24, "f16", seed=Lk)


@pytest.mark.parametrize("Lq", [1, 2, 31, 32, 33, 64, 65, 100, 129, 257, 300])
def test_attention_numbers_of_queries(Lq):
    attention_case(2, Lq, 37, 2, 2, 40, "bf16", seed=Lq)
    attention_case(1, Lq, 90, 2, 1, 17, "f32", seed=Lq)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (4, 2), (6, 1), (8, 8), (10, 5), (7, 1), (33, 1)])
def test_attention_heads(H, G):
    attention_case(2, 7, 45, H, G, 32, "bf16", seed=H)
    attention_case(1, 21, 33, H, G, 20, "f16", seed=H)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("q_lengths,lengths,mask", [
    ([50, 0, 7], None, None), (None, [0, 0, 0], None), (None, [100, 1, 64], None), (None, [-5, 200, 33], 0.5),
    ([50, 33, 99], [100, 65, 0], 0.9), (None, None, 0.1), (None, None, [[False] * 100, [True] * 100, [False] * 99 + [True]]),
    ([-1, 1, 50], [63, 64, 65], [[1, 0] * 50, [0] * 64 + [1] * 36, [0] * 63 + [2] + [0] * 36])])
def test_attention_masks(q_lengths, lengths, mask, dtype):
    mask = np.array(mask, dtype=np.uint8) if isinstance(mask, list) and not isinstance(mask[0][0], bool) else mask
    attention_case(3, 50, 100, 4, 2, 36, dtype, q_lengths, lengths, mask)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_attention_layouts(layout):
    attention_case(2, 20, 70, 4, 2, 24, "bf16", [20, 9], [70, 66], 0.8, layout)
    attention_case(2, 20, 40, 3, 3, 23, "f32", None, None, None, layout)
    attention_case(2, 20, 70, 4, 2, 33, "f16", None, [5, 70], None, layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,Lq,Lk,H,G,D", [(1, 300, 1500, 2, 2, 64), (2, 77, 2000, 8, 1, 96), (1, 1, 4100, 8, 2, 128),
                                           (40, 140, 200, 4, 4, 32), (1, 1200, 40, 2, 1, 48), (3, 513, 130, 16, 2, 128)])
def test_attention_larger(B, Lq, Lk, H, G, D, dtype):
    attention_case(B, Lq, Lk, H, G, D, dtype, seed=Lk)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_scores_far_apart(dtype):
    # rows that read one key alone, and a maximum that rises all along the keys
    attention_case(1, 40, 300, 2, 1, 64, dtype, spread=12.0)
    attention_case(1, 9, 400, 1, 1, 16, dtype, scale=3.0, spread=2.0)
    m = Make(3, dtype)
    q, k, v = torch.ones(1, 4, 1, 8, device="cuda", dtype=m.dtype), torch.zeros(1, 1000, 1, 8, device="cuda", dtype=m.dtype), m.act(1, 1000, 1, 8)
    k[0, :, 0, 0] = torch.arange(1000, device="cuda") / 4.0
    y, saved = seq.cross_attention_forward(q, k, v, scale=1.0, save=True)
    ry, rlse = oracle.cross_attention(host(q), host(k), host(v), 1.0)
    within(y, ry, (UNIT[y.dtype] + 2e-5) * np.abs(host(v)).max(), "y")
    within(saved[:4].view(1, 1, 4), rlse, 2e-5 * np.abs(rlse), "lse")


def test_attention_small_gradients_in_float16():
    # an upstream gradient at 2^-14 over 2000 keys: a score's gradient is some 2^-25, below float16's numbers
    attention_case(1, 60, 2000, 2, 1, 64, "f16", up=2.0 ** -14)
    # and a large one
    attention_case(1, 60, 300, 2, 1, 64, "f16", up=3000.0)


def test_attention_step_is_the_forward_of_one_token():
    m = Make(5, "bf16")
    q, k, v = m.act(3, 8, 64), m.act(3, 777, 2, 64), m.act(3, 777, 2, 64)
    mask = (m.f32(3, 777).cpu() < 1).cuda()
    kw = dict(lengths=i32([777, 0, 500]), mask=mask)
    y = seq.cross_attention_step(q, k, v, **kw)
    assert torch.equal(y, seq.cross_attention_forward(q[:, None], k, v, **kw)[0][:, 0])
    ry, _ = oracle.cross_attention(host(q)[:, None], host(k), host(v), lengths=[777, 0, 500], mask=mask.cpu().numpy())
    within(y, ry[:, 0], (2.0 ** -8 + 2e-5) * 4, "y")  # p @ |v| is below 4 with normal values
    assert not y[1].any()


def test_attention_nan_stays_in_its_row():
    m = Make(6, "bf16")
    q, k, v, gy = (m.act(1, 40, 2, 32) for _ in range(4))
    q[0, 3, 1] = float("nan")
    y, saved = seq.cross_attention_forward(q, k, v, save=True)
    bad = torch.isnan(y).all(-1)
    assert bad[0, 3, 1] and bad.sum() == 1 and torch.isnan(y).sum() == 32
    clean = q.clone()
    clean[0, 3, 1] = 0
    want, _ = seq.cross_attention_forward(clean, k, v)
    keep = ~bad
    assert torch.equal(y[keep], want[keep])
    g = seq.cross_attention_backward(gy, y, saved, q, k, v)
    assert torch.isnan(g.q).any(-1).sum() == 1 and not torch.isnan(g.k[:, :, 0]).any() and torch.isnan(g.k[:, :, 1]).all()


def test_attention_gradient_against_differences():
    m = Make(7)
    q, k, v, gy = m.f32(2, 6, 4, 8), m.f32(2, 9, 2, 8), m.f32(2, 9, 2, 8), m.f32(2, 6, 4, 8)
    kw = dict(lengths=i32([9, 5]), q_lengths=i32([4, 6]))
    y, saved = seq.cross_attention_forward(q, k, v, save=True, **kw)
    grads = seq.cross_attention_backward(gy, y, saved, q, k, v, **kw)
    for i, g in enumerate(grads):
        # along a direction: a step of 2^-6 has an error of its square times third derivatives of some 10 (1e-3), and float32's
        # 2^-24 of sums of some 100, over 2^-5 (2e-4)
        d = m.f32(*g.shape) / g.numel() ** 0.5
        ends = []
        for s in (2.0 ** -6, -2.0 ** -6):
            t = [q, k, v]
            t[i] = t[i] + s * d
            ends.append(float((seq.cross_attention_forward(*t, **kw)[0].double() * gy.double()).sum()))
        slope, want = (ends[0] - ends[1]) * 2.0 ** 5, float((g.double() * d.double()).sum())
        assert abs(slope - want) <= 3e-3 * (1 + abs(want)), "qkv"[i]


def test_attention_repeats_itself():
    m = Make(9, "f16")
    q, k, v, gy = m.act(2, 300, 4, 64), m.act(2, 900, 2, 64), m.act(2, 900, 2, 64), m.act(2, 300, 4, 64)
    runs = []
    for _ in range(3):
        y, saved = seq.cross_attention_forward(q, k, v, save=True)
        runs.append((y, saved, *seq.cross_attention_backward(gy, y, saved, q, k, v)))
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


# ----------------------------------------------------------------------------
# token log probabilities
# ----------------------------------------------------------------------------
def logprobs_check(z, tokens, top, temperature, glogp=None, gentropy=None, gtop=None, hz=None):
    hz = host(z) if hz is None else hz
    ht = None if tokens is None else tokens.cpu().numpy()
    r = seq.token_logprobs_forward(z, tokens, top=top, temperature=temperature)
    logp, entropy, idx, values = oracle.token_logprobs(hz, ht, top, temperature)
    tol = lambda ref: 1e-5 * (1 + np.abs(np.where(np.isfinite(ref), ref, 0)))  # noqa: E731
    within(r.entropy, entropy, tol(entropy), "entropy")
    assert (r.logp is None) == (tokens is None)
    if tokens is not None:
        within(r.logp, logp, tol(logp), "logp")
    if top:
        assert r.idx.dtype == torch.int32 and np.array_equal(r.idx.cpu().numpy(), idx)
        within(r.top, values, tol(values), "top")
    else:
        assert r.idx is None and r.top is None
    if glogp is None and gentropy is None and gtop is None:
        return r
    gz = seq.token_logprobs_backward(r.stats, z, tokens, glogp=glogp, gentropy=gentropy, idx=r.idx, gtop=gtop,
                                     temperature=temperature)
    hg = [host(g) for g in (glogp, gentropy, gtop)]
    want = oracle.token_logprobs_backward(hz, ht, hg[0], hg[1], idx, hg[2], temperature)
    parts, flushed = np.zeros(hz.shape), np.zeros(hz.shape)
    for i in range(len(hz)):
        l = oracle._log_softmax(hz[i], temperature)
        p = np.exp(l)
        a = sum(np.abs(g[i]).sum() for g in (hg[0], hg[2]) if g is not None)
        h = 0 if hg[1] is None else np.abs(hg[1][i])
        by = a + h * (np.abs(np.where(p > 0, l, 0)) + np.log(len(l)))
        parts[i], flushed[i] = np.where(p > 0, p * by, 0), 2.0 ** -126 * by
        if hg[0] is not None and 0 <= ht[i] < len(l):
            parts[i, ht[i]] += np.abs(hg[0][i])
        if hg[2] is not None:
            parts[i, idx[i]] += np.abs(hg[2][i])
    within(gz, want, (4e-5 * np.nan_to_num(parts) + np.nan_to_num(flushed)) / temperature, "gz")
    over = z.clone()
    same = seq.token_logprobs_backward(r.stats, over, tokens, glogp=glogp, gentropy=gentropy, idx=r.idx, gtop=gtop,
                                       temperature=temperature, gz=over)
    assert same is over and torch.equal(over.view(torch.uint8), gz.view(torch.uint8)) or torch.isnan(gz).any()
    return r


def logprobs_case(R, V, K, dtype="f32", temperature=1.0, seed=0, spread=2.0, layout="dense"):
    print(f"logprobs R={R} V={V} K={K} {dtype} temperature={temperature} {layout}", flush=True)
    m = Make(seed, dtype)
    z = m.act(R, V, scale=spread)
    if layout == "slice":
        z = torch.full((R, V + 9), float("nan"), dtype=z.dtype, device="cuda")[:, 3:V + 3].copy_(z)
    tokens = m.ints(-1, V, R)
    logprobs_check(z, tokens, K, temperature, m.f32(R), m.f32(R), m.f32(R, K) if K else None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,K", [(1, 1), (2, 1), (3, 3), (7, 0), (8, 5), (63, 20), (128, 128), (129, 128), (200, 64), (512, 100),
                                 (513, 128), (1000, 128), (2049, 1), (4097, 40), (8192, 128), (8200, 10), (20011, 128),
                                 (32000, 64), (32769, 33)])
def test_logprobs_vocabularies(V, K, dtype):
    logprobs_case(3, V, K, dtype, seed=V)


@pytest.mark.parametrize("dtype,V", [("f32", 40001), ("bf16", 70001), ("f16", 131077), ("bf16", 65536), ("f32", 200003)])
def test_logprobs_long_rows(dtype, V):
    logprobs_case(2, V, 50, dtype, 0.7)


@pytest.mark.parametrize("dtype,V,K", [("f32", 9000, 20), ("bf16", 17000, 128), ("f16", 33000, 7), ("f32", 33000, 3),
                                       ("bf16", 66000, 20)])
def test_logprobs_many_rows(dtype, V, K):
    print(f"logprobs many rows {dtype} {V} {K}", flush=True)
    m = Make(V, dtype)
    z, tokens = m.act(600, V, scale=2.0), m.ints(-1, V, 600)
    some = [0, 1, 299, 598, 599]
    up = [m.f32(600), m.f32(600), m.f32(600, K)]
    r = seq.token_logprobs_forward(z, tokens, top=K, temperature=1.5)
    gz = seq.token_logprobs_backward(r.stats, z, tokens, *up[:2], r.idx, up[2], 1.5)
    logp, entropy, idx, values = oracle.token_logprobs(host(z[some]), tokens[some].cpu().numpy(), K, 1.5)
    within(r.logp[some], logp, 1e-5 * (1 + np.abs(logp)), "logp")
    within(r.entropy[some], entropy, 1e-5 * (1 + np.abs(entropy)), "entropy")
    assert np.array_equal(r.idx[some].cpu().numpy(), idx)
    within(r.top[some], values, 1e-5 * (1 + np.abs(values)), "top")
    want = oracle.token_logprobs_backward(host(z[some]), tokens[some].cpu().numpy(), *(host(u[some]) for u in up[:2]), idx,
                                          host(up[2][some]), 1.5)
    # a term is at most (|glogp| + sum |gtop| + |gentropy| (|l| + log V)) p, and at a named place 1 in p's place
    most = 4e-5 * sum(np.abs(host(u[some])).reshape(5, -1).sum(1) for u in up)[:, None] * 30
    p = np.exp((host(z[some]) - host(z[some]).max(1, keepdims=True)) / 1.5)
    p = p / p.sum(1, keepdims=True)
    for i in range(5):
        p[i, idx[i]] = 1
        p[i, tokens[some[i]]] = 1
    within(gz[some], want, most * p, "gz")


@pytest.mark.parametrize("layout", ["slice"])
def test_logprobs_layouts(layout):
    logprobs_case(5, 1001, 20, "bf16", layout=layout)
    logprobs_case(5, 333, 20, "f32", 2.0, layout=layout)


@pytest.mark.parametrize("temperature", [0.05, 0.5, 1.0, 7.0])
def test_logprobs_temperatures(temperature):
    logprobs_case(4, 3000, 16, "f32", temperature)
    logprobs_case(4, 3000, 16, "f16", temperature)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 600, 5000, 30000, 70000])
def test_logprobs_equal_logits(V, dtype):
    # rows of one value, of two, of few, and sorted either way: many candidates, told apart by place
    K = min(V, 100)
    t = DTYPES[dtype]
    v = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), (v % 2).float(), (v % 7 * -0.5), v / 1000.0, -v / 1000.0,
            torch.where(v == V - 1, 1.0, torch.where(v % 3 == 0, -0.0, 0.0)), torch.full((V,), torch.finfo(t).min, device="cuda"),
            torch.where(v > V - 3, 2.0, torch.finfo(t).min)]
    z = torch.stack([r.float() for r in rows]).to(t)
    print(f"equal logits V={V} {dtype}", flush=True)
    tokens = i32([0, V - 1, 2, 3, 4, V - 1, 1, 0])
    m = Make(V)
    logprobs_check(z, tokens, K, 1.0, m.f32(8), m.f32(8), m.f32(8, K))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("V", [40, 3000, 40000, 140000])
def test_logprobs_values_at_the_edge(V, dtype):
    inf, nan = float("inf"), float("nan")
    m = Make(V, dtype)
    z = m.act(8, V)
    z[0, 1:] = -inf  # one place left
    z[1, ::2] = -inf
    z[2] = -inf  # nothing left
    z[3, 5] = inf
    z[4, 7] = nan
    z[5] = nan
    z[6, [3, 30, 11]] = nan
    z[6, :3] = -inf
    z[7, V // 2:] = -inf
    print(f"edge values V={V} {dtype}", flush=True)
    tokens = i32([0, 1, 2, 3, 4, 5, V, V - 1])
    K = 20
    r = seq.token_logprobs_forward(z, tokens, top=K)
    logp, entropy, idx, values = oracle.token_logprobs(host(z), tokens.cpu().numpy(), K)
    tol = lambda ref: 1e-5 * (1 + np.abs(np.where(np.isfinite(ref), ref, 0)))  # noqa: E731
    within(r.logp, logp, tol(logp), "logp")
    within(r.entropy, entropy, tol(entropy), "entropy")
    assert np.array_equal(r.idx.cpu().numpy(), idx)
    within(r.top, values, tol(values), "top")
    # gradients of the rows that have them, and of a token past the vocabulary
    fine = [0, 1, 7]
    g = torch.ones(8, device="cuda")
    gz = seq.token_logprobs_backward(r.stats, z, tokens, glogp=g, gentropy=g)
    want = oracle.token_logprobs_backward(host(z[fine]), tokens[fine].cpu().numpy(), np.ones(3), np.ones(3))
    within(gz[fine], want, 4e-5 * 30, "gz")
    assert torch.isnan(gz[6]).all()
    # rows that are not asked for are 0, whatever they hold
    g[:] = 0
    assert not seq.token_logprobs_backward(r.stats, z, tokens, glogp=g, gentropy=g).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [40, 3000, 40000, 140000])
def test_logprobs_far_from_zero(V, dtype):
    # the products of logits and log2(e) lose bits, and more than a binade's worth past 2^24; the differences do not.  The last
    # two rows go that far from chunk to chunk, up and down.
    m, most = Make(V, dtype), 15 if dtype == "f16" else 70
    far = [2.0 ** 10, -(2.0 ** 13), 2.0 ** min(19, most), 2.0 ** min(24, most), -(2.0 ** min(34, most)), 2.0 ** most]
    grow = 2.0 ** (torch.arange(V, device="cuda") * (most / V))
    rows = [(m.f32(V) * 2 + f).clamp(-65000.0, 65000.0) if dtype == "f16" else m.f32(V) * 2 + f for f in far] + [grow, -grow]
    z = torch.stack(rows).to(DTYPES[dtype])
    print(f"far from zero V={V} {dtype}", flush=True)
    logprobs_check(z, i32([0, V - 1, 2, 3, 4, V - 1, V - 1, 0]), 20, 1.0, m.f32(8), m.f32(8), m.f32(8, 20))
    logprobs_check(z, i32([0, V - 1, 2, 3, 4, V - 1, V - 1, 0]), 0, 0.125, m.f32(8), m.f32(8))


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_logprobs_extreme_temperatures(V):
    # the hottest is a uniform distribution over the places that are there, the coldest one of the largest logits
    m = Make(V)
    z = m.act(4, V)
    z[1, ::2] = -float("inf")
    z[2, :V // 2] = -float("inf")
    z[3, 1:] = -float("inf")
    print(f"extreme temperatures V={V}", flush=True)
    for temperature in (8e37, 1e33, 2e-38):
        logprobs_check(z, i32([0, 1, V - 1, 0]), 5, temperature)


def test_logprobs_parts():
    m = Make(2, "bf16")
    z = m.act(6, 500)
    logprobs_check(z, None, 0, 1.0, gentropy=m.f32(6))
    logprobs_check(z, None, 9, 1.0, gtop=m.f32(6, 9))
    logprobs_check(z, m.ints(0, 500, 6), 0, 1.0, glogp=m.f32(6))
    # the same place named by the token and twice by idx: their gradients add up; an absent entry has none
    r = seq.token_logprobs_forward(z, i32([7] * 6))
    idx, g = i32([[7, 3, 7, -1]] * 6), m.f32(6, 4)
    gz = seq.token_logprobs_backward(r.stats, z, i32([7] * 6), glogp=g[:, 0].contiguous(), idx=idx, gtop=g)
    want = oracle.token_logprobs_backward(host(z), [7] * 6, host(g[:, 0]), None, idx.cpu().numpy(), host(g))
    within(gz, want, 4e-5 * 10, "gz")


def test_logprobs_gradient_against_differences():
    m = Make(4)
    z, tokens, gl, gh = m.f32(3, 50), m.ints(0, 50, 3), m.f32(3), m.f32(3)
    r = seq.token_logprobs_forward(z, tokens, temperature=1.3)
    g = seq.token_logprobs_backward(r.stats, z, tokens, glogp=gl, gentropy=gh, temperature=1.3)
    d = m.f32(3, 50) / 12
    ends = []
    for s in (2.0 ** -6, -2.0 ** -6):
        e = seq.token_logprobs_forward(z + s * d, tokens, temperature=1.3)
        ends.append(float((e.logp.double() * gl.double() + e.entropy.double() * gh.double()).sum()))
    slope, want = (ends[0] - ends[1]) * 2.0 ** 5, float((g.double() * d.double()).sum())
    assert abs(slope - want) <= 2e-3 * (1 + abs(want))  # the step's square times third derivatives of some units


# ----------------------------------------------------------------------------
# together, on other streams, in graphs
# ----------------------------------------------------------------------------
def read_image(q, k, v, pos_q, pos_k, freqs, w, tokens, up):
    """Queries and keys with their positions, the attention, a projection to codes, their scores, and all the way back."""
    kw = dict(sections=(4, 6, 6))
    rq, rk = seq.rotary_forward(q, pos_q, freqs, **kw), seq.rotary_forward(k, pos_k, freqs, **kw)
    y, saved = seq.cross_attention_forward(rq, rk, v, save=True)
    flat = y.flatten(0, 1).flatten(1)
    z = flat @ w
    r = seq.token_logprobs_forward(z, tokens, top=8)
    gz = seq.token_logprobs_backward(r.stats, z, tokens, glogp=up, gentropy=up)
    gy = (gz @ w.t().contiguous()).view(y.shape)
    g = seq.cross_attention_backward(gy, y, saved, rq, rk, v)
    return [y, r.logp, r.entropy, r.idx, r.top, seq.rotary_backward(g.q, pos_q, freqs, **kw),
            seq.rotary_backward(g.k, pos_k, freqs, **kw), g.v]


def reading_inputs(m, B=2, Lq=20, Lk=64, H=4, G=2, D=40, V=300):
    image = torch.stack(torch.meshgrid(torch.arange(1), torch.arange(8), torch.arange(Lk // 8), indexing="ij"), -1)
    text = torch.arange(Lq)[None, :, None].expand(B, Lq, 3) + 9
    return dict(q=m.act(B, Lq, H, D), k=m.act(B, Lk, G, D), v=m.act(B, Lk, G, D),
                pos_q=text.to(torch.int32).contiguous().cuda(), pos_k=image.view(Lk, 3).to(torch.int32).cuda(),
                freqs=torch.exp(-m.f32(16).abs()), w=m.act(H * D, V, scale=0.2), tokens=m.ints(0, V, B * Lq), up=m.f32(B * Lq))


def test_reading_an_image_against_autograd():
    m = Make(11)
    x = reading_inputs(m)
    got = read_image(**x)
    q, k, v = (x[n].double().cpu().requires_grad_() for n in "qkv")

    def turn(t, pos):
        axis = torch.tensor([0] * 4 + [1] * 6 + [2] * 6)
        a = (pos.cpu().double()[..., axis] * x["freqs"].cpu().double())[..., None, :]
        u, w, rest = t[..., :16], t[..., 16:32], t[..., 32:]
        return torch.cat([u * a.cos() - w * a.sin(), u * a.sin() + w * a.cos(), rest], -1)

    rq, rk = turn(q, x["pos_q"]).transpose(1, 2), turn(k, x["pos_k"]).transpose(1, 2).repeat_interleave(2, 1)
    p = torch.softmax(rq @ rk.transpose(-1, -2) * 40 ** -0.5, -1)
    y = (p @ v.transpose(1, 2).repeat_interleave(2, 1)).transpose(1, 2)
    l = torch.log_softmax(y.flatten(0, 1).flatten(1) @ x["w"].cpu().double(), 1)
    logp = l.gather(1, x["tokens"].cpu().long()[:, None])[:, 0]
    entropy = -(l.exp() * l).sum(1)
    up = x["up"].cpu().double()
    grads = torch.autograd.grad([logp, entropy], (q, k, v), [up, up])
    # float32 throughout: each step within 2e-5 of its sums (torch's product among them), ten of them
    for name, a, b in zip(("y", "logp", "entropy", "gq", "gk", "gv"), (got[0], got[1], got[2], *got[5:]),
                          (y, logp, entropy, *grads)):
        b = b.detach().numpy()
        within(a, b, 2e-4 * np.abs(b).max(), name)
    assert np.array_equal(got[3].cpu().numpy(), l.topk(8, 1).indices.numpy())


def test_reading_on_another_stream():
    x = reading_inputs(Make(12, "bf16"))
    want = read_image(**x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = read_image(**x)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_reading_in_a_graph():
    x = reading_inputs(Make(13, "bf16"), Lk=512, V=70000)
    read_image(**x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = read_image(**x)
    for seed in (14, 15, 16):
        fresh = reading_inputs(Make(seed, "bf16"), Lk=512, V=70000)
        for n in x:
            x[n].copy_(fresh[n])
        graph.replay()
        torch.cuda.synchronize()
        want = read_image(**x)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_two_captured_steps_share_no_workspace():
    m = Make(17, "f16")
    k, v = m.act(2, 3000, 2, 64), m.act(2, 3000, 2, 64)
    qs = [m.act(2, 8, 64) for _ in range(2)]
    want = [seq.cross_attention_step(q, k, v) for q in qs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(seq.cross_attention_step(q, k, v))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


# ----------------------------------------------------------------------------
# refusals
# ----------------------------------------------------------------------------
def test_refusals():
    m = Make(1, "bf16")
    x, pos, f = m.act(2, 3, 4, 16), m.ints(0, 9, 2, 3, 2), m.f32(8)
    with pytest.raises(ValueError, match="sections"):
        seq.rotary_forward(x, pos, f, sections=(4, 5))
    with pytest.raises(ValueError, match="positions"):
        seq.rotary_forward(x, pos, f, sections=(8,))
    with pytest.raises(ValueError, match="positions"):
        seq.rotary_forward(x, pos.long(), f, sections=(4, 4))
    with pytest.raises(ValueError, match="freqs"):
        seq.rotary_forward(x, pos, f.double(), sections=(4, 4))
    with pytest.raises(FdcError, match="pairs of channels"):
        seq.rotary_forward(x, m.ints(0, 9, 2, 3, 1), m.f32(9))
    with pytest.raises(FdcError, match="y shares memory with x"):
        seq.rotary_forward(x[:, :2], pos[:, :2], f, sections=(4, 4), y=x[:, 1:])
    with pytest.raises(ValueError, match="GPU tensor"):
        seq.rotary_forward(x.cpu(), pos, f, sections=(4, 4))
    q, k = m.act(2, 3, 4, 16), m.act(2, 5, 2, 16)
    with pytest.raises(ValueError, match="k has shape"):
        seq.cross_attention_forward(q, k[..., :8], k[..., :8])
    with pytest.raises(ValueError, match="v has shape"):
        seq.cross_attention_forward(q, k, k[:, :4])
    with pytest.raises(FdcError, match="multiple of G"):
        seq.cross_attention_forward(q[:, :, :3], k, k)
    with pytest.raises(FdcError, match="scale"):
        seq.cross_attention_forward(q, k, k, scale=0.0)
    with pytest.raises(ValueError, match="mask"):
        seq.cross_attention_forward(q, k, k, mask=torch.ones(2, 5, device="cuda"))
    with pytest.raises(ValueError, match="mask has shape"):
        seq.cross_attention_forward(q, k, k, mask=torch.ones(2, 4, device="cuda", dtype=torch.bool))
    with pytest.raises(FdcError, match="y shares memory with q"):
        seq.cross_attention_forward(q, k, k, y=q)
    with pytest.raises(FdcError, match="at most 128"):
        seq.cross_attention_step(m.act(1, 1, 129), m.act(1, 4, 1, 129), m.act(1, 4, 1, 129))
    y, saved = seq.cross_attention_forward(q, k, k, save=True)
    with pytest.raises(ValueError, match="saved has shape"):
        seq.cross_attention_backward(y, y, saved[:-1], q, k, k)
    z = m.act(3, 20)
    with pytest.raises(FdcError, match="K must be"):
        seq.token_logprobs_forward(z, top=21)
    with pytest.raises(FdcError, match="at most 128"):
        seq.token_logprobs_forward(m.act(3, 200), top=129)
    with pytest.raises(FdcError, match="tau"):
        seq.token_logprobs_forward(z, temperature=0.0)
    with pytest.raises(ValueError, match="tokens"):
        seq.token_logprobs_forward(z, tokens=torch.zeros(3, device="cuda", dtype=torch.int64))
    r = seq.token_logprobs_forward(z)
    with pytest.raises(FdcError, match="no gradient"):
        seq.token_logprobs_backward(r.stats, z)
    with pytest.raises(FdcError, match="glogp without tokens"):
        seq.token_logprobs_backward(r.stats, z, glogp=m.f32(3))
    with pytest.raises(ValueError, match="gtop goes with idx"):
        seq.token_logprobs_backward(r.stats, z, gtop=m.f32(3, 2))
    with pytest.raises(FdcError, match="gz shares memory"):
        seq.token_logprobs_backward(r.stats[:2], z[:2], gentropy=m.f32(2), gz=z[1:])
