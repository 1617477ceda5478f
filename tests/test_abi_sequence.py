"""Host-side tests of the sequence operators' C ABI: sizes, strides and parts are checked, with the
documented status, before the GPU is touched (every call here returns from host-side validation), and
again against the host-sanitized build."""

import ctypes
import os
import shutil
import subprocess
import sys

import pytest

from paper_2106_12736_amd import _lib
from paper_2106_12736_amd._lib import (FDC_EINVAL, FDC_EUNSUPPORTED, FDC_EWORKSPACE, FDC_OK, ConvArgs, DistillArgs,
                                       NormArgs, NormGrads, ScanArgs, ScanGrads, Tokens)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000  # never dereferenced: validation fails first


def _size(name, *args):
    n = ctypes.c_size_t()
    st = _lib.status(name, *args, ctypes.byref(n))
    return n.value if st == FDC_OK else -st


def _with(cls, base, **change):
    a = cls(*base.values())
    for k, v in change.items():
        setattr(a, k, v)
    return a


def _tok(L, D):
    return Tokens(P, L * D, D)


CONV = dict(dtype=1, B=2, L=6, D=8, n=4, silu=1, x=_tok(6, 8), y=_tok(6, 8), w=P, bias=P, state=None, new_state=None,
            lengths=None)
SCAN = dict(dtype=1, B=2, L=6, D=8, N=4, G=2, softplus=1, x=_tok(6, 8), dt=_tok(6, 8), gate=_tok(6, 8), Bm=_tok(6, 8),
            Cm=_tok(6, 8), y=_tok(6, 8), A=P, skip=P, dt_bias=P, h0=None, h_last=None, lengths=None)
NORM = dict(dtype=1, D=8, act=2, R=5, eps=1e-6, x=P, f=P, gate=P, x_stride=8, f_stride=8, gate_stride=8, scale=P,
            w_post=P, w_pre=P)
DIST = dict(dtype=1, V=8, K=2, R=5, tau=1.0, alpha=0.5, z=P, z_stride=8, idx=P, teacher=P, labels=P, weight=P)


@pytest.mark.parametrize("change,want", [
    ({"dtype": 3}, FDC_EINVAL), ({"B": 0}, FDC_EINVAL), ({"L": 0}, FDC_EINVAL), ({"D": -1}, FDC_EINVAL),
    ({"n": 0}, FDC_EINVAL), ({"n": 9}, FDC_EUNSUPPORTED), ({"B": 65536}, FDC_EUNSUPPORTED),
    ({"w": None}, FDC_EINVAL), ({"x": Tokens(None, 48, 8)}, FDC_EINVAL), ({"x": Tokens(P, 48, -8)}, FDC_EINVAL),
    ({"x": Tokens(P, 48, 1 << 26)}, FDC_EUNSUPPORTED), ({"y": Tokens(P, 48, 7)}, FDC_EINVAL),
    ({"y": Tokens(P, 47, 8)}, FDC_EINVAL), ({"y": Tokens(P, 8, 15)}, FDC_EINVAL), ({"y": Tokens(None, 0, 0)}, FDC_EINVAL),
    ({"L": 1 << 28, "D": 1 << 20}, FDC_EUNSUPPORTED),
])
def test_conv_refuses(change, want):
    assert _lib.status("fdc_causal_conv_forward", _with(ConvArgs, CONV, **change), None) == want
    assert _lib.last_error()


def test_conv_backward_refuses():
    a, none = _with(ConvArgs, CONV), Tokens(None, 0, 0)
    back = lambda gy, gx, gw, ws, n: _lib.status("fdc_causal_conv_backward", a, gy, gx, gw, None, ws, n, None)  # noqa: E731
    need = _size("fdc_causal_conv_workspace_size", 1, 2, 6, 8, 4)
    assert need > 0
    assert back(none, _tok(6, 8), P, P, need) == FDC_EINVAL
    assert back(_tok(6, 8), Tokens(P, 48, 0), P, P, need) == FDC_EINVAL
    assert back(_tok(6, 8), _tok(6, 8), P, P, need - 1) == FDC_EWORKSPACE
    assert back(_tok(6, 8), _tok(6, 8), P, None, need) == FDC_EWORKSPACE
    assert back(_tok(6, 8), _tok(6, 8), P, P + 4, need) == FDC_EINVAL
    assert back(_tok(6, 8), none, None, None, 0) == FDC_OK  # nothing is asked for, nothing enqueued
    assert _size("fdc_causal_conv_workspace_size", 1, 2, 6, 8, 9) == -FDC_EUNSUPPORTED


@pytest.mark.parametrize("change,want", [
    ({"dtype": -1}, FDC_EINVAL), ({"N": 0}, FDC_EINVAL), ({"N": 65}, FDC_EUNSUPPORTED), ({"G": 3}, FDC_EINVAL),
    ({"G": 0}, FDC_EINVAL), ({"A": None}, FDC_EINVAL), ({"dt": Tokens(None, 0, 0)}, FDC_EINVAL),
    ({"Bm": Tokens(None, 0, 0)}, FDC_EINVAL), ({"y": Tokens(P, 48, 0)}, FDC_EINVAL),
    ({"gate": Tokens(P, -1, 8)}, FDC_EINVAL), ({"h0": P, "h_last": P}, FDC_EINVAL),
    ({"B": 4096, "D": 1 << 15, "N": 16}, FDC_EUNSUPPORTED),
])
def test_scan_refuses(change, want):
    assert _lib.status("fdc_scan_forward", _with(ScanArgs, SCAN, **change), None, P, 1 << 40, None) == want
    assert _lib.last_error()


def test_scan_saved_and_workspaces():
    assert _size("fdc_scan_saved_size", 2, 33, 8, 4) == 2 * 3 * 8 * 4 * 4
    assert _size("fdc_scan_saved_size", 2, 33, 8, 65) == -FDC_EUNSUPPORTED
    # a long sequence of few channels is cut into chunks, whose states take a workspace
    f = ctypes.c_size_t()
    assert _lib.status("fdc_scan_workspace_size", 1, 8192, 64, 16, 1, ctypes.byref(f), None) == FDC_OK and f.value > 0
    x = _tok(8192, 64)
    a = _with(ScanArgs, SCAN, B=1, L=8192, D=64, N=16, G=1, x=x, dt=x, gate=x, y=x, Bm=_tok(8192, 16), Cm=_tok(8192, 16))
    assert _lib.status("fdc_scan_forward", a, None, None, 0, None) == FDC_EWORKSPACE
    assert _lib.status("fdc_scan_forward", a, P + 4, P, f.value, None) == FDC_EINVAL


def test_scan_backward_and_step_refuse():
    t, none = _tok(6, 8), Tokens(None, 0, 0)
    a = _with(ScanArgs, SCAN)
    g = lambda **c: _with(ScanGrads, dict(gy=t, gx=t, gdt=t, ggate=t, gBm=t, gCm=t, gA=P, gskip=P, gdt_bias=P), **c)  # noqa: E731
    back = lambda gr, saved=P, n=1 << 40: _lib.status("fdc_scan_backward", a, saved, gr, P, n, None)  # noqa: E731
    assert back(g(), saved=None) == FDC_EINVAL
    for name in ("gy", "gx", "gdt", "ggate", "gBm", "gCm"):
        assert back(g(**{name: none})) == FDC_EINVAL, name
    for name in ("gA", "gskip", "gdt_bias"):
        assert back(g(**{name: None})) == FDC_EINVAL, name
    assert back(g(), n=16) == FDC_EWORKSPACE
    step = lambda **c: _lib.status("fdc_scan_step", _with(ScanArgs, SCAN, **c), None)  # noqa: E731
    assert step(h0=P, h_last=P) == FDC_EINVAL  # L = 6
    assert step(L=1, h0=P) == FDC_EINVAL
    assert step(L=1, h0=P, h_last=P, lengths=P) == FDC_EINVAL


@pytest.mark.parametrize("change,want", [
    ({"dtype": 7}, FDC_EINVAL), ({"R": 0}, FDC_EINVAL), ({"D": 0}, FDC_EINVAL), ({"D": 8193}, FDC_EUNSUPPORTED),
    ({"act": 3}, FDC_EINVAL), ({"eps": 0.0}, FDC_EINVAL), ({"eps": float("nan")}, FDC_EINVAL), ({"x": None}, FDC_EINVAL),
    ({"f": None}, FDC_EINVAL), ({"x_stride": -8}, FDC_EINVAL), ({"w_pre": None}, FDC_EINVAL),
])
def test_norm_refuses(change, want):
    a = _with(NormArgs, NORM, **change)
    assert _lib.status("fdc_block_norm_forward", a, P, 8, P, 8, P, None) == want


def test_norm_outputs_and_backward_refuse():
    a = _with(NormArgs, NORM)
    assert _lib.status("fdc_block_norm_forward", a, P, 7, P, 8, P, None) == FDC_EINVAL
    assert _lib.status("fdc_block_norm_forward", a, P, 8, None, 8, P, None) == FDC_EINVAL
    base = dict(gout=P, gn=P, gx=P, gf=P, ggate=P, gout_stride=8, gn_stride=8, gx_stride=8, gf_stride=8, ggate_stride=8,
                gscale=P, gw_post=P, gw_pre=P)
    need = _size("fdc_block_norm_workspace_size", 5, 8)
    back = lambda args, stats=P, n=need, **c: _lib.status("fdc_block_norm_backward", args, stats,  # noqa: E731
                                                          _with(NormGrads, base, **c), P, n, None)
    assert need > 0 and back(a, n=need - 1) == FDC_EWORKSPACE
    assert back(a, stats=None) == FDC_EINVAL
    assert back(a, gout=None, gn=None) == FDC_EINVAL
    assert back(a, gx_stride=4) == FDC_EINVAL
    assert back(_with(NormArgs, NORM, gate=None)) == FDC_EINVAL  # ggate without a gate
    assert back(_with(NormArgs, NORM, w_pre=None)) == FDC_EINVAL  # gn without w_pre


@pytest.mark.parametrize("change,want", [
    ({"dtype": 9}, FDC_EINVAL), ({"R": 0}, FDC_EINVAL), ({"V": 0}, FDC_EINVAL), ({"K": 0}, FDC_EINVAL),
    ({"K": 1025}, FDC_EUNSUPPORTED), ({"tau": 0.0}, FDC_EINVAL), ({"tau": float("inf")}, FDC_EINVAL),
    ({"alpha": -0.1}, FDC_EINVAL), ({"alpha": float("nan")}, FDC_EINVAL), ({"z": None}, FDC_EINVAL),
    ({"idx": None}, FDC_EINVAL), ({"teacher": None}, FDC_EINVAL), ({"z_stride": -1}, FDC_EINVAL),
    ({"V": (1 << 24) + 1}, FDC_EUNSUPPORTED),
])
def test_distill_refuses(change, want):
    a = _with(DistillArgs, DIST, **change)
    assert _lib.status("fdc_distill_forward", a, P, P, P, 1 << 40, None) == want
    assert _lib.status("fdc_distill_backward", a, P, P, P, 8, None) == want
    assert _lib.status("fdc_distill_forward_backward", a, P, P, P, P, 8, P, 1 << 40, None) == want


def test_distill_outputs_refuse():
    a = _with(DistillArgs, DIST)
    need = _size("fdc_distill_workspace_size", 1, 5, 8)
    assert _lib.status("fdc_distill_forward", a, P, P, None, need, None) == FDC_EWORKSPACE
    assert _lib.status("fdc_distill_forward", a, None, P, P, need, None) == FDC_EINVAL
    assert _lib.status("fdc_distill_backward", a, P, P, P, 7, None) == FDC_EINVAL
    assert _lib.status("fdc_distill_backward", a, P, P, P, 9, None) == FDC_EINVAL  # z's memory, another stride
    assert _lib.status("fdc_distill_forward_backward", a, P, P, P, None, 8, P, need, None) == FDC_EINVAL


def test_null_arguments():
    for name, rest in (("fdc_causal_conv_forward", (None,)), ("fdc_scan_step", (None,)),
                       ("fdc_block_norm_forward", (P, 8, P, 8, P, None)), ("fdc_distill_forward", (P, P, P, 8, None))):
        assert _lib.status(name, None, *rest) == FDC_EINVAL, name


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
