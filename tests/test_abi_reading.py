"""Host-side tests of the reading operators' C ABI (rotary positions, cross attention, token log probabilities): sizes,
strides, parts and shared memory are checked, with the documented status, before the GPU is touched, and again
against the host-sanitized build.  (Each call here is refused, so that none reaches the GPU.)"""

import ctypes
import os
import random
import shutil
import subprocess
import sys

import pytest

from paper_2106_12736_amd import _lib
from paper_2106_12736_amd._lib import (FDC_EINVAL, FDC_EUNSUPPORTED, FDC_EWORKSPACE, FDC_OK, CrossAttentionArgs,
                                       CrossAttentionGrads, Heads, RotaryArgs, TokenLogprobsArgs)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x100000  # never dereferenced: validation fails first


def _with(cls, base, **change):
    a = cls(*base.values())
    for k, v in change.items():
        setattr(a, k, v)
    return a


def _heads(at, B, L, H, D):
    return Heads(P * at, L * H * D, H * D, D)


def _pairs(*n):
    return (ctypes.c_int * 4)(*n)


ROT = dict(dtype=1, B=2, L=6, H=3, D=16, axes=2, interleaved=0, inverse=0, pairs=_pairs(4, 4), x=_heads(1, 2, 6, 3, 16),
           y=_heads(2, 2, 6, 3, 16), positions=P, pos_batch_stride=12, pos_token_stride=2, freqs=P, lengths=None)
ATT = dict(dtype=1, B=2, Lq=6, Lk=9, H=4, G=2, D=16, scale=0.25, q=_heads(1, 2, 6, 4, 16), k=_heads(2, 2, 9, 2, 16),
           v=_heads(3, 2, 9, 2, 16), y=_heads(4, 2, 6, 4, 16), q_lengths=None, lengths=None, mask=None, mask_stride=0)
LOG = dict(dtype=1, V=50, K=4, R=5, tau=1.0, z=P, z_stride=50, tokens=P)


@pytest.mark.parametrize("change,want", [
    ({"dtype": 3}, FDC_EINVAL), ({"B": 0}, FDC_EINVAL), ({"L": 0}, FDC_EINVAL), ({"H": 0}, FDC_EINVAL), ({"D": 0}, FDC_EINVAL),
    ({"B": 65536}, FDC_EUNSUPPORTED), ({"H": 65536}, FDC_EUNSUPPORTED), ({"D": 1025}, FDC_EUNSUPPORTED),
    ({"axes": 0}, FDC_EINVAL), ({"axes": 5}, FDC_EINVAL), ({"axes": 3}, FDC_EINVAL), ({"pairs": _pairs(4, -1)}, FDC_EINVAL),
    ({"pairs": _pairs(4, 5)}, FDC_EINVAL), ({"pairs": _pairs(2 ** 31 - 1, 2 ** 31 - 1)}, FDC_EINVAL),
    ({"positions": None}, FDC_EINVAL), ({"freqs": None}, FDC_EINVAL), ({"pos_batch_stride": -1}, FDC_EINVAL),
    ({"pos_token_stride": -2}, FDC_EINVAL), ({"pos_token_stride": 1 << 25}, FDC_EUNSUPPORTED),
    ({"x": Heads(None, 0, 0, 0)}, FDC_EINVAL), ({"y": Heads(None, 0, 0, 0)}, FDC_EINVAL),
    ({"x": Heads(P, 288, -48, 16)}, FDC_EINVAL), ({"x": Heads(P, 288, 48, 1 << 30)}, FDC_EUNSUPPORTED),
    ({"x": Heads(P, 1 << 46, 48, 16)}, FDC_EUNSUPPORTED), ({"y": Heads(2 * P, 288, 48, 15)}, FDC_EINVAL),
    ({"y": Heads(2 * P, 287, 48, 16)}, FDC_EINVAL), ({"y": Heads(2 * P, 0, 48, 16)}, FDC_EINVAL),
    ({"L": 1 << 28, "B": 16}, FDC_EUNSUPPORTED),
])
def test_rotary_refuses(change, want):
    assert _lib.status("fdc_rotary", _with(RotaryArgs, ROT, **change), None) == want
    assert _lib.last_error()


@pytest.mark.parametrize("change,want", [
    ({"dtype": -1}, FDC_EINVAL), ({"B": 0}, FDC_EINVAL), ({"Lq": 0}, FDC_EINVAL), ({"Lk": 0}, FDC_EINVAL), ({"H": 0}, FDC_EINVAL),
    ({"G": 0}, FDC_EINVAL), ({"H": 5}, FDC_EINVAL), ({"D": 0}, FDC_EINVAL), ({"D": 129}, FDC_EUNSUPPORTED),
    ({"B": 65536}, FDC_EUNSUPPORTED), ({"Lk": (1 << 28) + 1}, FDC_EUNSUPPORTED), ({"Lq": 1 << 28, "H": 1 << 15}, FDC_EUNSUPPORTED),
    ({"B": 65535, "H": 65534, "G": 65534}, FDC_EUNSUPPORTED), ({"B": 60000, "Lk": 1 << 28, "H": 60000, "G": 60000}, FDC_EUNSUPPORTED),
    ({"scale": 0.0}, FDC_EINVAL), ({"scale": -1.0}, FDC_EINVAL), ({"scale": float("nan")}, FDC_EINVAL),
    ({"scale": float("inf")}, FDC_EINVAL), ({"q": Heads(None, 0, 0, 0)}, FDC_EINVAL), ({"k": Heads(None, 0, 0, 0)}, FDC_EINVAL),
    ({"v": Heads(P, -1, 32, 16)}, FDC_EINVAL), ({"y": Heads(4 * P, 384, 64, 8)}, FDC_EINVAL),
    ({"k": Heads(P, 288, 1 << 25, 16)}, FDC_EUNSUPPORTED), ({"mask": P, "mask_stride": -1}, FDC_EINVAL),
    ({"mask": P, "mask_stride": 1 << 46}, FDC_EUNSUPPORTED),
])
def test_attention_refuses(change, want):
    a = _with(CrossAttentionArgs, ATT, **change)
    assert _lib.status("fdc_cross_attention_forward", a, None, P, 1 << 40, None) == want
    assert _lib.last_error()


def test_attention_sizes_and_workspaces():
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    size = lambda *a: (_lib.status("fdc_cross_attention_saved_size", *a, ctypes.byref(n)), n.value)  # noqa: E731
    assert size(0, 2, 6, 4, 16) == (FDC_OK, 2 * 6 * 4 * 4)  # the logarithms alone
    assert size(1, 2, 6, 4, 16) == (FDC_OK, 2 * 6 * 4 * (4 + 2 * 16))
    assert size(1, 1, 1, 1, 3) == (FDC_OK, 16 + 16)
    assert size(1, 1, 1, 1, 129)[0] == FDC_EUNSUPPORTED
    query = lambda *a: _lib.status("fdc_cross_attention_workspace_size", *a, ctypes.byref(n), ctypes.byref(m))  # noqa: E731
    # a long cache read by few rows is cut into runs, and so are the sums over many rows
    assert query(1, 1, 1, 1 << 20, 8, 2, 128) == FDC_OK and n.value > 0
    assert query(1, 1, 64, 64, 2, 2, 64) == FDC_OK and m.value >= 64 * 2 * 8
    assert query(1, 1, 1, 1 << 20, 8, 3, 128) == FDC_EINVAL
    assert _lib.status("fdc_cross_attention_workspace_size", 1, 1, 1, 64, 8, 2, 128, None, None) == FDC_OK
    a = _with(CrossAttentionArgs, ATT, B=1, Lq=1, Lk=1 << 20, H=8, G=2, D=128, q=_heads(1, 1, 1, 8, 128),
              k=Heads(1 << 40, 1 << 28, 256, 128), v=Heads(1 << 41, 1 << 28, 256, 128), y=_heads(2, 1, 1, 8, 128))
    assert query(1, 1, 1, 1 << 20, 8, 2, 128) == FDC_OK
    call = lambda ws, size, saved=None: _lib.status("fdc_cross_attention_forward", a, saved, ws, size, None)  # noqa: E731
    assert call(None, 0) == FDC_EWORKSPACE and call(P, n.value - 1) == FDC_EWORKSPACE
    assert call(P + 4, n.value) == FDC_EINVAL and call(P, n.value, P + 8) == FDC_EINVAL


def test_attention_backward_refuses():
    g = dict(gy=_heads(5, 2, 6, 4, 16), gq=_heads(6, 2, 6, 4, 16), gk=_heads(7, 2, 9, 2, 16), gv=_heads(8, 2, 9, 2, 16))
    m = ctypes.c_size_t()
    assert _lib.status("fdc_cross_attention_workspace_size", 1, 2, 6, 9, 4, 2, 16, None, ctypes.byref(m)) == FDC_OK

    def say(saved=P << 8, size=1 << 30, args=None, **change):
        st = _lib.status("fdc_cross_attention_backward", _with(CrossAttentionArgs, ATT, **(args or {})), saved,
                         _with(CrossAttentionGrads, g, **change), P << 9, size, None)
        return st, _lib.last_error()

    assert say(saved=None)[0] == FDC_EINVAL and say(saved=P + 4)[0] == FDC_EINVAL
    assert say(size=m.value - 1)[0] == FDC_EWORKSPACE
    for name in ("gy", "gq", "gk", "gv"):
        assert say(**{name: Heads(None, 0, 0, 0)})[0] == FDC_EINVAL, name
    assert say(gq=Heads(6 * P, 384, 64, 8))[0] == FDC_EINVAL
    assert say(gq=g["gy"]) == (FDC_EINVAL, "gq shares memory with gy")
    assert say(gq=ATT["y"]) == (FDC_EINVAL, "gq shares memory with y")
    assert say(gk=ATT["k"]) == (FDC_EINVAL, "gk shares memory with k")
    assert say(gv=g["gk"]) == (FDC_EINVAL, "gv shares memory with gk")
    # keys and values side by side in one buffer, as their projection leaves them, are apart
    both = lambda off: Heads(P * 7 + 2 * off, 9 * 64, 64, 16)  # noqa: E731
    assert say(gk=both(0), gv=both(32), size=0)[0] == FDC_EWORKSPACE
    assert say(gk=both(0), gv=both(31), size=0) == (FDC_EINVAL, "gv shares memory with gk")


def _elements(offset, B, L, H, D, bs, ts, hs):
    return {offset + b * bs + t * ts + h * hs + d for b in range(B) for t in range(L) for h in range(H) for d in range(D)}


def test_shared_memory_of_heads():
    # gq against k, of every order of strides, by sets of element addresses; what is apart is refused for its workspace
    refused = accepted = 0
    rng = random.Random(2)
    for _ in range(4000):
        B, L, H, D = (rng.randint(1, 3) for _ in range(4))
        order, strides, extent = rng.sample(range(3), 3), [0, 0, 0], D
        for axis in order:
            strides[axis] = extent + rng.randint(0, 4)
            extent = ((B, L, H)[axis] - 1) * strides[axis] + extent
        shift = rng.randint(-2 * extent, 2 * extent)
        over = bool(_elements(0, B, L, H, D, *strides) & _elements(shift, B, L, H, D, *strides))
        a = CrossAttentionArgs(1, B, L, L, H, H, D, 1.0, Heads(P << 4, *strides), Heads(P + 2 * shift, *strides),
                               Heads(P << 5, *strides), Heads(P << 9, *strides), None, None, None, 0)
        g = CrossAttentionGrads(Heads(P << 6, *strides), Heads(P, *strides), Heads(P << 7, *strides), Heads(P << 8, *strides))
        st = _lib.status("fdc_cross_attention_backward", a, P << 10, g, None, 0, None)
        assert st == (FDC_EINVAL if over else FDC_EWORKSPACE), (B, L, H, D, strides, shift, _lib.last_error())
        if over:
            assert _lib.last_error() == "gq shares memory with k"
        refused, accepted = refused + over, accepted + (not over)
    assert refused > 500 and accepted > 500


def test_rotary_over_its_input():
    # the whole of x is allowed (refused later, for its size), a part of it is not
    x = Heads(P, 288, 48, 16)
    fine = _with(RotaryArgs, ROT, x=x, y=x, freqs=None)
    assert _lib.status("fdc_rotary", fine, None) == FDC_EINVAL and "freqs" in _lib.last_error()
    for y in (Heads(P + 2, 288, 48, 16), Heads(P + 96, 288, 48, 16), Heads(P - 30, 288, 48, 16), Heads(P, 300, 50, 16)):
        assert _lib.status("fdc_rotary", _with(RotaryArgs, ROT, x=x, y=y), None) == FDC_EINVAL
        assert _lib.last_error() == "y shares memory with x"


@pytest.mark.parametrize("change,want", [
    ({"dtype": 9}, FDC_EINVAL), ({"R": 0}, FDC_EINVAL), ({"V": 0}, FDC_EINVAL), ({"K": -1}, FDC_EINVAL), ({"K": 51}, FDC_EINVAL),
    ({"V": 1000, "K": 129, "z_stride": 1000}, FDC_EUNSUPPORTED), ({"tau": 0.0}, FDC_EINVAL), ({"tau": float("nan")}, FDC_EINVAL),
    ({"tau": float("inf")}, FDC_EINVAL), ({"tau": 4e-39}, FDC_EINVAL), ({"tau": 2e38}, FDC_EINVAL), ({"z": None}, FDC_EINVAL), ({"z_stride": -1}, FDC_EINVAL),
    ({"V": (1 << 24) + 1}, FDC_EUNSUPPORTED), ({"R": 1 << 26}, FDC_EUNSUPPORTED), ({"R": 1 << 25, "V": 1 << 20}, FDC_EUNSUPPORTED),
])
def test_logprobs_refuses(change, want):
    a = _with(TokenLogprobsArgs, LOG, **change)
    assert _lib.status("fdc_token_logprobs_forward", a, P, P, P, P, P, P, 1 << 60, None) == want
    assert _lib.status("fdc_token_logprobs_backward", a, P, P, P, P, P, P << 4, max(a.V, 50), None) == want


def test_logprobs_parts_refuse():
    a, none = _with(TokenLogprobsArgs, LOG), _with(TokenLogprobsArgs, LOG, tokens=None)
    fwd = lambda a, *outs: _lib.status("fdc_token_logprobs_forward", a, *outs, P, 1 << 40, None)  # noqa: E731
    assert fwd(none, P, P, P, P, P) == FDC_EINVAL and fwd(a, None, P, P, P, P) == FDC_EINVAL  # logp goes with tokens
    assert fwd(a, P, P, None, P, P) == FDC_EINVAL and fwd(a, P, P, P, None, P) == FDC_EINVAL
    assert fwd(_with(TokenLogprobsArgs, LOG, K=0), P, P, P, P, P) == FDC_EINVAL
    assert fwd(_with(TokenLogprobsArgs, LOG, K=0, tokens=None), None, None, None, None, None) == FDC_EINVAL
    back = lambda a, stats, gl, gh, idx, gt, gz=P << 4, gs=50: _lib.status(  # noqa: E731
        "fdc_token_logprobs_backward", a, stats, gl, gh, idx, gt, gz, gs, None)
    assert back(a, None, P, P, P, P) == FDC_EINVAL and back(a, P, P, P, P, P, None) == FDC_EINVAL
    assert back(a, P, None, None, P, None) == FDC_EINVAL and back(none, P, P, P, P, P) == FDC_EINVAL
    assert back(a, P, P, P, None, P) == FDC_EINVAL and back(a, P, P, P, P, P, P << 4, 49) == FDC_EINVAL
    for gz, stride in ((P + 2, 50), (P + 100, 50), (P, 51)):
        assert back(a, P, P, P, P, P, gz, stride) == FDC_EINVAL and _lib.last_error() == "gz shares memory with z"


def test_logprobs_workspace():
    n = ctypes.c_size_t()
    size = lambda *a: (_lib.status("fdc_token_logprobs_workspace_size", *a, ctypes.byref(n)), n.value)  # noqa: E731
    assert size(1, 4096, 32000, 64) == (FDC_OK, 0)
    st, need = size(1, 2, 1 << 20, 64)
    assert st == FDC_OK and need > 0
    assert size(1, 2, 50, 51)[0] == FDC_EINVAL
    assert _lib.status("fdc_token_logprobs_workspace_size", 1, 2, 50, 5, None) == FDC_EINVAL
    a = _with(TokenLogprobsArgs, LOG, R=2, V=1 << 20, K=64, z_stride=1 << 20)
    assert _lib.status("fdc_token_logprobs_forward", a, P, P, P, P, P, P, need - 1, None) == FDC_EWORKSPACE
    assert _lib.status("fdc_token_logprobs_forward", a, P, P, P, P, P, P + 8, need, None) == FDC_EINVAL


def test_null_arguments():
    for name, rest in (("fdc_rotary", (None,)), ("fdc_cross_attention_forward", (P, P, 8, None)),
                       ("fdc_token_logprobs_forward", (P, P, P, P, P, P, 8, None))):
        assert _lib.status(name, None, *rest) == FDC_EINVAL, name
    a = _with(CrossAttentionArgs, ATT)
    assert _lib.status("fdc_cross_attention_backward", a, P, None, P, 8, None) == FDC_EINVAL


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc is needed to build the sanitized library")
@pytest.mark.skipif("FDC_LIBRARY" in os.environ, reason="this is the run against another build")
def test_under_host_sanitizers():
    from paper_2106_12736_amd import build

    env = dict(os.environ, FDC_LIBRARY=build.build_host_sanitized(verbose=False), LD_PRELOAD=build.asan_runtime(),
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert "passed" in r.stdout


@pytest.mark.parametrize("B,Lq,Lk,H,G,D", [(65535, 1, 256, 65, 1, 128), (32768, 1, 64, 128, 2, 64), (65535, 4, 9, 60, 4, 32),
                                           (1, 1 << 20, 40, 64, 1, 64)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_what_attends_can_be_saved(dtype, B, Lq, Lk, H, G, D):
    # the size of what is saved has no number of key heads: that of the call decides
    n = ctypes.c_size_t()
    assert _lib.status("fdc_cross_attention_workspace_size", dtype, B, Lq, Lk, H, G, D, None, None) == FDC_OK
    assert _lib.status("fdc_cross_attention_saved_size", dtype, B, Lq, H, D, ctypes.byref(n)) == FDC_OK, _lib.last_error()
    rows, pieces = B * Lq * H, lambda n: (n + 15) // 16 * 16  # each part in pieces of 16 bytes
    assert n.value == pieces(4 * rows) + (0 if dtype == 0 else pieces(2 * rows * D))


def test_what_is_too_large_cannot_be_saved():
    n = ctypes.c_size_t()
    size = lambda *a: _lib.status("fdc_cross_attention_saved_size", *a, ctypes.byref(n))  # noqa: E731
    assert size(1, 65535, 1 << 20, 1, 128) == FDC_EUNSUPPORTED and size(1, 65535, 1 << 28, 65535, 128) == FDC_EUNSUPPORTED
    assert size(1, 1, 1, 65536, 8) == FDC_EUNSUPPORTED and size(1, 1, 1, 0, 8) == FDC_EINVAL
    assert size(1, 0, 1, 1, 8) == FDC_EINVAL and size(3, 1, 1, 1, 8) == FDC_EINVAL
    assert _lib.status("fdc_cross_attention_saved_size", 1, 1, 1, 1, 8, None) == FDC_EINVAL


@pytest.mark.parametrize("scale", [2.5e38, 3.4e38])
def test_scales_whose_exponents_leave_float32_are_refused(scale):
    # scale log2(e) enters the kernels; an unaligned `saved` is what the call is refused for otherwise
    a = _with(CrossAttentionArgs, ATT, scale=scale)
    assert _lib.status("fdc_cross_attention_forward", a, P + 8, P, 1 << 40, None) == FDC_EINVAL
    assert "scale" in _lib.last_error()
    g = CrossAttentionGrads(*(_heads(5 + i, 2, 6 if i < 2 else 9, 4 if i < 2 else 2, 16) for i in range(4)))
    assert _lib.status("fdc_cross_attention_backward", a, P + 8, g, P, 1 << 40, None) == FDC_EINVAL
    assert "scale" in _lib.last_error()
    a.scale = 2.2e38
    assert _lib.status("fdc_cross_attention_forward", a, P + 8, P, 1 << 40, None) == FDC_EINVAL
    assert "saved" in _lib.last_error()
