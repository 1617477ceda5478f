"""Torch-facing wrappers of libfdc's sequence operators: the block of a sequence network and
the loss it is trained with, on tokens of D channels.

  causal_conv_*   causal convolution of each channel with its own short kernel (and SiLU)
  scan_*          selective state space scan
  block_norm_*    norm of a block's output, gate, residual scale, and the norm before the next block
  distill_*       loss against a teacher's top logits and labels

and what it reads an image's tokens and scores its answers with:

  rotary_*            rotary positions of several axes
  cross_attention_*   attention to states of another length
  token_logprobs_*    log probabilities of given tokens, entropy, top alternatives

Activations are float32, bfloat16 or float16, of shape [B, L, D] (or [B, D] for one token; [B, L, H, D] or [B, H, D]
where they have heads) with any strides whose last dimension is dense; parameters, states and losses are float32 and contiguous.
Every call runs on the current stream of the current device, which the tensors have to be on, and
allocates its outputs and workspace there; an output that is given is other memory than the inputs
unless a function says that it may be the same.  include/fdc.h defines each operation.
"""

import ctypes
from collections import namedtuple
from functools import lru_cache

import torch

from . import _lib
from ._lib import (ConvArgs, CrossAttentionArgs, CrossAttentionGrads, DistillArgs, Heads, NormArgs, NormGrads,
                   RotaryArgs, ScanArgs, TokenLogprobsArgs, Tokens, call)
from .layers import _ptr, _stream

_DTYPES = {torch.float32: _lib.DTYPE_F32, torch.bfloat16: _lib.DTYPE_BF16, torch.float16: _lib.DTYPE_F16}
_ACTS = {"none": 0, "sigmoid": 1, "silu": 2}
_ABSENT = Tokens(None, 0, 0)

ScanGradients = namedtuple("ScanGradients", "x dt A B C skip gate dt_bias")
NormGradients = namedtuple("NormGradients", "x f gate scale w_post w_pre")
AttentionGradients = namedtuple("AttentionGradients", "q k v")
TokenLogprobs = namedtuple("TokenLogprobs", "logp entropy idx top stats")


# Calls on single tokens are bound by this file's own work, so a tensor that passes its check costs one
# comparison chain, and what is wrong with another is found out afterwards.
def _kind(t, name):
    """The fdc_dtype of an activation on the current device."""
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16 (got {t.dtype})")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    return d


def _wrong(t, dtype, device, shape, name):
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device} (got {t.dtype} on {t.device})")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _strides(t, ref, shape, name):
    """The strides of an activation of ref's type and device, of this shape, its last dimension dense."""
    if t is not ref and not (t.dtype == ref.dtype and t.get_device() == ref.get_device() and t.shape == shape):
        _wrong(t, ref.dtype, ref.device, shape, name)
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}'s last dimension must be dense")
    return s


def _tokens(t, ref, shape, name):
    if t is None:
        return _ABSENT
    s = _strides(t, ref, shape, name)
    return Tokens(t.data_ptr(), s[0], s[1] if len(s) > 2 else 0)


def _tokens_groups(t, ref, shape, name):
    """B or C of a scan, [..., G, N] with the groups of a token side by side."""
    s = _strides(t, ref, shape, name)
    if s[-2] != shape[-1] and shape[-2] > 1:
        raise ValueError(f"{name}'s groups must be dense")
    return Tokens(t.data_ptr(), s[0], s[1] if len(s) > 3 else 0)


def _heads(t, ref, shape, name):
    """[B, L, heads, D], or [B, heads, D] of one token."""
    s = _strides(t, ref, shape, name)
    return Heads(t.data_ptr(), s[0], s[1], s[2]) if len(s) == 4 else Heads(t.data_ptr(), s[0], 0, s[1])


def _rows(t, ref, shape, name):
    """Pointer and row stride of an optional [R, D] activation."""
    if t is None:
        return None, 0
    return t.data_ptr(), _strides(t, ref, shape, name)[0]


def _dense(t, dtype, ref, shape, name):
    """The pointer of an optional dense parameter, state, loss or list of integers."""
    if t is None:
        return None
    if t.dtype == dtype and t.get_device() == ref.get_device() and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    _wrong(t, dtype, ref.device, shape, name)
    raise ValueError(f"{name} must be contiguous")


def _f32(t, ref, shape, name):
    return _dense(t, torch.float32, ref, shape, name)


def _i32(t, ref, shape, name):
    return _dense(t, torch.int32, ref, shape, name)


def _empty(shape, ref, dtype=None):
    return ref.new_empty(shape, dtype=dtype)


@lru_cache(maxsize=4096)
def _bytes(name, *sizes, which=0, of=1):
    """What a workspace query (a function of sizes alone) says: its output `which` of `of`."""
    n = [ctypes.c_size_t() for _ in range(of)]
    call(name, *sizes, *(ctypes.byref(v) for v in n))
    return n[which].value


def _scratch(nbytes, ref):
    """Pointer and size of a workspace, and the tensor that keeps it (until the call has been enqueued)."""
    if nbytes == 0:
        return None, 0, None
    t = ref.new_empty(nbytes, dtype=torch.uint8)
    return t.data_ptr(), nbytes, t


def _like(t):
    """An output of t's shape, in its layout where that is dense; its last dimension is."""
    if t is None:
        return None
    out = torch.empty_like(t)
    # rows that overlap (windows one element apart) leave torch no order of the dimensions
    return out if out.dim() == 0 or out.stride(-1) == 1 or t.shape[-1] == 1 else t.new_empty(t.shape)


# ----------------------------------------------------------------------------
# causal convolution
# ----------------------------------------------------------------------------
def _conv_args(x, w, bias, silu, state, lengths, y, new_state):
    if x.dim() not in (2, 3):
        raise ValueError(f"x must be [B, L, D] or [B, D] (got {tuple(x.shape)})")
    dt = _kind(x, "x")
    shape = x.shape
    B, D = shape[0], shape[-1]
    if w.dim() != 2:
        raise ValueError(f"w must be [D, taps] (got {tuple(w.shape)})")
    n = w.shape[1]
    kept = (B, n - 1, D)
    return ConvArgs(dt, B, shape[1] if len(shape) == 3 else 1, D, n, silu, _tokens(x, x, shape, "x"),
                    _tokens(y, x, shape, "y"), _f32(w, x, (D, n), "w"), _f32(bias, x, (D,), "bias"),
                    _dense(state, x.dtype, x, kept, "state"), _dense(new_state, x.dtype, x, kept, "new_state"),
                    _i32(lengths, x, (B,), "lengths"))


def causal_conv_forward(x, w, bias=None, silu=False, state=None, lengths=None, last=False, y=None):
    """x [B, L, D], w [D, taps], bias [D] -> (y, new_state): y[t] = bias + sum_j w[j] x[t - taps + 1 + j],
    with SiLU if asked (fdc_causal_conv_forward).  state [B, taps - 1, D]: the tokens before x;
    new_state: the last ones, if `last` is asked for, else None."""
    y = _like(x) if y is None else y
    a = _conv_args(x, w, bias, silu, state, lengths, y, None)
    new_state = _empty((a.B, a.n - 1, a.D), x) if last else None
    a.new_state = _ptr(new_state)
    call("fdc_causal_conv_forward", a, _stream())
    return y, new_state


def causal_conv_step(x, w, state, bias=None, silu=False, new_state=None, y=None):
    """One token x [B, D] of every sequence -> (y, new_state); the state is updated in place unless
    new_state is given, and y may be x itself."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D] (got {tuple(x.shape)})")
    y = _like(x) if y is None else y
    new_state = state if new_state is None else new_state
    call("fdc_causal_conv_forward", _conv_args(x, w, bias, silu, state, None, y, new_state), _stream())
    return y, new_state


def causal_conv_backward(gy, x, w, bias=None, silu=False, state=None, lengths=None, need_gx=True, need_gw=True):
    """-> (gx, gw, gbias) from gy (fdc_causal_conv_backward); gbias is None without a bias."""
    a = _conv_args(x, w, bias, silu, state, lengths, None, None)
    gx = _like(x) if need_gx else None
    gw = _like(w) if need_gw else None
    gbias = _like(bias) if need_gw else None
    need = _bytes("fdc_causal_conv_workspace_size", a.dtype, a.B, a.L, a.D, a.n) if need_gw else 0
    ws, size, keep = _scratch(need, x)
    call("fdc_causal_conv_backward", a, _tokens(gy, x, x.shape, "gy"), _tokens(gx, x, x.shape, "gx"), _ptr(gw),
         _ptr(gbias), ws, size, _stream())
    return gx, gw, gbias


# ----------------------------------------------------------------------------
# selective scan
# ----------------------------------------------------------------------------
def _scan_args(x, dt, A, B, C, skip, gate, dt_bias, softplus, h0, h_last, lengths, y):
    kind = _kind(x, "x")
    shape = x.shape
    if len(shape) not in (2, 3):
        raise ValueError(f"x must be [B, L, D] or [B, D] (got {tuple(shape)})")
    nb, D = shape[0], shape[-1]
    if A.dim() != 2 or B.dim() != x.dim() + 1:
        raise ValueError(f"A must be [D, N] and B {'[B, L, G, N]' if x.dim() == 3 else '[B, G, N]'} "
                         f"(got {tuple(A.shape)}, {tuple(B.shape)})")
    N, G = A.shape[1], B.shape[-2]
    shared, state = (nb, G, N) if len(shape) == 2 else (nb, shape[1], G, N), (nb, D, N)
    return ScanArgs(kind, nb, shape[1] if len(shape) == 3 else 1, D, N, G, softplus, _tokens(x, x, shape, "x"),
                    _tokens(dt, x, shape, "dt"), _tokens(gate, x, shape, "gate"), _tokens_groups(B, x, shared, "B"),
                    _tokens_groups(C, x, shared, "C"), _tokens(y, x, shape, "y"), _f32(A, x, (D, N), "A"),
                    _f32(skip, x, (D,), "skip"), _f32(dt_bias, x, (D,), "dt_bias"), _f32(h0, x, state, "h0"),
                    _f32(h_last, x, state, "h_last"), _i32(lengths, x, (nb,), "lengths"))


def scan_forward(x, dt, A, B, C, skip=None, gate=None, dt_bias=None, softplus=True, h0=None, lengths=None,
                 last=False, save=False, y=None):
    """Selective scan (fdc_scan_forward) of x, dt, gate [B, L, D] with A [D, N], B, C [B, L, G, N], skip and
    dt_bias [D] from the state h0 [B, D, N] -> (y, h_last, saved): the state after the last token if `last`
    is asked for, and what scan_backward needs if `save` is; else None.  y may be x, dt or gate
    itself (which scan_backward would need)."""
    if x.dim() != 3:
        raise ValueError(f"x must be [B, L, D] (got {tuple(x.shape)})")
    y = _like(x) if y is None else y
    a = _scan_args(x, dt, A, B, C, skip, gate, dt_bias, softplus, h0, None, lengths, y)
    h_last = _empty((a.B, a.D, a.N), x, torch.float32) if last else None
    a.h_last = _ptr(h_last)
    saved = _empty((_bytes("fdc_scan_saved_size", a.B, a.L, a.D, a.N) // 4,), x, torch.float32) if save else None
    ws, size, keep = _scratch(_bytes("fdc_scan_workspace_size", a.B, a.L, a.D, a.N, a.G, which=0, of=2), x)
    call("fdc_scan_forward", a, _ptr(saved), ws, size, _stream())
    return y, h_last, saved


def scan_backward(gy, saved, x, dt, A, B, C, skip=None, gate=None, dt_bias=None, softplus=True, lengths=None):
    """Gradients of scan_forward's inputs (None for those that are not given) from gy and what it saved."""
    a = _scan_args(x, dt, A, B, C, skip, gate, dt_bias, softplus, None, None, lengths, None)
    _f32(saved, x, (_bytes("fdc_scan_saved_size", a.B, a.L, a.D, a.N) // 4,), "saved")
    ws, size, keep = _scratch(_bytes("fdc_scan_workspace_size", a.B, a.L, a.D, a.N, a.G, which=1, of=2), x)
    g = ScanGradients(*(_like(t) for t in (x, x, A)), _empty(B.shape, x), _empty(B.shape, x),
                      *(_like(t) for t in (skip, None if gate is None else x, dt_bias)))
    s = _lib.ScanGrads(_tokens(gy, x, x.shape, "gy"), _tokens(g.x, x, x.shape, "gx"), _tokens(g.dt, x, x.shape, "gdt"),
                       _tokens(g.gate, x, x.shape, "ggate"), _tokens_groups(g.B, x, B.shape, "gB"),
                       _tokens_groups(g.C, x, B.shape, "gC"), _ptr(g.A), _ptr(g.skip), _ptr(g.dt_bias))
    call("fdc_scan_backward", a, _ptr(saved), s, ws, size, _stream())
    return g


def scan_step(x, dt, A, B, C, h, skip=None, gate=None, dt_bias=None, softplus=True, h_new=None, y=None):
    """One token of every sequence (fdc_scan_step): x, dt, gate [B, D], B, C [B, G, N], state h [B, D, N] ->
    (y, h_new); the state is updated in place unless h_new is given, and y may be x, dt or gate itself."""
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D] (got {tuple(x.shape)})")
    y = _like(x) if y is None else y
    h_new = h if h_new is None else h_new
    call("fdc_scan_step", _scan_args(x, dt, A, B, C, skip, gate, dt_bias, softplus, h, h_new, None, y), _stream())
    return y, h_new


# ----------------------------------------------------------------------------
# block norm
# ----------------------------------------------------------------------------
def _norm_args(x, f, gate, scale, w_post, w_pre, act, eps):
    dt = _kind(x, "x")
    if x.dim() != 2:
        raise ValueError(f"x must be [tokens, D] (got {tuple(x.shape)})")
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)} (got {act!r})")
    shape = x.shape
    R, D = shape
    (xp, xs), (fp, fs), (gp, gs) = _rows(x, x, shape, "x"), _rows(f, x, shape, "f"), _rows(gate, x, shape, "gate")
    return NormArgs(dt, D, _ACTS[act], R, eps, xp, fp, gp, xs, fs, gs, _f32(scale, x, (D,), "scale"),
                    _f32(w_post, x, (D,), "w_post"), _f32(w_pre, x, (D,), "w_pre"))


def block_norm_forward(x, f=None, gate=None, scale=None, w_post=None, w_pre=None, act="silu", eps=1e-6):
    """x, f, gate [tokens, D] -> (out, n, stats) (fdc_block_norm_forward): out = x + scale act(gate) rms(f; w_post)
    and n = rms(out; w_pre).  Without f, out is x itself; n is None without w_pre."""
    a = _norm_args(x, f, gate, scale, w_post, w_pre, act, eps)
    out = x if f is None else _like(x)
    n = None if w_pre is None else _like(x)
    stats = _empty((a.R, 2), x, torch.float32)
    call("fdc_block_norm_forward", a, None if f is None else out.data_ptr(), out.stride(0), _ptr(n),
         0 if n is None else n.stride(0), stats.data_ptr(), _stream())
    return out, n, stats


def block_norm_backward(gout, gn, stats, x, f=None, gate=None, scale=None, w_post=None, w_pre=None, act="silu",
                        eps=1e-6):
    """Gradients of block_norm_forward's inputs (None for those that are not given) from the gradients of out
    and n (either may be None) and the forward's stats."""
    a = _norm_args(x, f, gate, scale, w_post, w_pre, act, eps)
    _f32(stats, x, (a.R, 2), "stats")
    (gop, gos), (gnp, gns) = _rows(gout, x, x.shape, "gout"), _rows(gn, x, x.shape, "gn")
    rows = _like(x)
    g = NormGradients(rows, *(None if t is None else _like(rows) for t in (f, gate)),
                      *(_like(t) for t in (scale, w_post, w_pre)))
    ws, size, keep = _scratch(_bytes("fdc_block_norm_workspace_size", a.R, a.D), x)
    s = NormGrads(gop, gnp, _ptr(g.x), _ptr(g.f), _ptr(g.gate), gos, gns, *(rows.stride(0),) * 3,
                  _ptr(g.scale), _ptr(g.w_post), _ptr(g.w_pre))
    call("fdc_block_norm_backward", a, _ptr(stats), s, ws, size, _stream())
    return g


# ----------------------------------------------------------------------------
# distillation
# ----------------------------------------------------------------------------
def _distill_args(z, idx, teacher, temperature, labels, alpha, weight):
    dt = _kind(z, "z")
    if z.dim() != 2 or idx.dim() != 2:
        raise ValueError(f"z must be [rows, vocabulary] and idx [rows, K] (got {tuple(z.shape)}, {tuple(idx.shape)})")
    R, K = z.shape[0], idx.shape[1]
    return DistillArgs(dt, z.shape[1], K, R, temperature, alpha, *_rows(z, z, z.shape, "z"),
                       _i32(idx, z, (R, K), "idx"), _dense(teacher, z.dtype, z, (R, K), "teacher"),
                       _i32(labels, z, (R,), "labels"), _f32(weight, z, (R,), "weight"))


def _distill_ws(a, ref):
    return _scratch(_bytes("fdc_distill_workspace_size", a.dtype, a.R, a.V), ref)


def distill_forward(z, idx, teacher, temperature=1.0, labels=None, alpha=1.0, weight=None):
    """Loss of each row of z [rows, V] against the teacher's logits [rows, K] at the places idx [rows, K] (int32,
    -1: absent) and, with labels [rows] (int32, -1: none), 1 - alpha of the cross-entropy
    (fdc_distill_forward) -> (loss [rows], stats)."""
    a = _distill_args(z, idx, teacher, temperature, labels, alpha, weight)
    loss, stats = _empty((a.R,), z, torch.float32), _empty((a.R, 5), z, torch.float32)
    ws, size, keep = _distill_ws(a, z)
    call("fdc_distill_forward", a, _ptr(loss), _ptr(stats), ws, size, _stream())
    return loss, stats


def distill_backward(gloss, stats, z, idx, teacher, temperature=1.0, labels=None, alpha=1.0, weight=None, gz=None):
    """Gradient of z from that of the loss [rows] and distill_forward's stats (gz may be z itself)."""
    a = _distill_args(z, idx, teacher, temperature, labels, alpha, weight)
    gz = _like(z) if gz is None else gz
    gp, gs = _rows(gz, z, z.shape, "gz")
    call("fdc_distill_backward", a, _f32(stats, z, (a.R, 5), "stats"), _f32(gloss, z, (a.R,), "gloss"), gp, gs,
         _stream())
    return gz


def distill_forward_backward(gloss, z, idx, teacher, temperature=1.0, labels=None, alpha=1.0, weight=None, gz=None):
    """Loss and gradient in one call, for a gradient of the loss that is known beforehand -> (loss, gz)."""
    a = _distill_args(z, idx, teacher, temperature, labels, alpha, weight)
    loss, stats = _empty((a.R,), z, torch.float32), _empty((a.R, 5), z, torch.float32)
    gz = _like(z) if gz is None else gz
    gp, gs = _rows(gz, z, z.shape, "gz")
    ws, size, keep = _distill_ws(a, z)
    call("fdc_distill_forward_backward", a, _f32(gloss, z, (a.R,), "gloss"), _ptr(loss), _ptr(stats), gp, gs, ws,
         size, _stream())
    return loss, gz


# ----------------------------------------------------------------------------
# rotary positions
# ----------------------------------------------------------------------------
@lru_cache(maxsize=4096)
def _pairs(sections, freqs_shape):
    """The number of axes and the pairs of each, as the C ABI takes them."""
    if sections is None and len(freqs_shape) == 1:
        sections = tuple(freqs_shape)
    if sections is None or not 1 <= len(sections) <= 4 or tuple(freqs_shape) != (sum(sections),):
        raise ValueError(f"sections are the pairs of 1 to 4 axes, and freqs has one a pair (got {sections}, {tuple(freqs_shape)})")
    return len(sections), (ctypes.c_int * 4)(*sections)


def _rotary(x, positions, freqs, sections, interleaved, lengths, y, inverse):
    dt = _kind(x, "x")
    shape = x.shape
    if len(shape) == 4:
        B, L, H, D = shape
    elif len(shape) == 3:
        (B, H, D), L = shape, 1
    else:
        raise ValueError(f"x must be [B, L, H, D] or [B, H, D] (got {tuple(shape)})")
    axes, pairs = _pairs(sections if sections is None else tuple(sections), freqs.shape)
    # [L, axes] of [B, L, H, D]: the same for every sequence
    want = (B, axes) if len(shape) == 3 else (L, axes) if positions.dim() == 2 else (B, L, axes)
    if positions.shape != want or positions.dtype != torch.int32 or positions.get_device() != x.get_device():
        _wrong(positions, torch.int32, x.device, want, "positions")
    s = positions.stride()
    batch, token = (s[0], 0) if len(shape) == 3 else (0, s[0]) if len(want) == 2 else (s[0], s[1])
    if s[-1] != 1 and axes > 1:
        raise ValueError("positions' last dimension must be dense")
    y = _like(x) if y is None else y
    call("fdc_rotary", RotaryArgs(dt, B, L, H, D, axes, interleaved, inverse, pairs, _heads(x, x, shape, "x"),
                                  _heads(y, x, shape, "y"), positions.data_ptr(), batch, token,
                                  _f32(freqs, x, freqs.shape, "freqs"), _i32(lengths, x, (B,), "lengths")), _stream())
    return y


def rotary_forward(x, positions, freqs, sections=None, interleaved=False, lengths=None, y=None):
    """x [B, L, H, D] (or [B, H, D], one token) with each pair of channels turned by position * frequency (fdc_rotary) -> y.
    positions [B, L, axes] or [L, axes] ([B, axes]) int32; sections: the number of pairs of each axis (None: one
    axis); freqs [pairs] float32, in the sections' order.  Pairs are the channels (i, pairs + i), or (2 i, 2 i + 1) if
    interleaved; other channels are copied.  y may be x itself."""
    return _rotary(x, positions, freqs, sections, interleaved, lengths, y, False)


def rotary_backward(gy, positions, freqs, sections=None, interleaved=False, lengths=None, gx=None):
    """-> gx from gy: the turn back (gx may be gy itself)."""
    return _rotary(gy, positions, freqs, sections, interleaved, lengths, gx, True)


# ----------------------------------------------------------------------------
# cross attention
# ----------------------------------------------------------------------------
def _attention_args(q, k, v, scale, q_lengths, lengths, mask, y):
    dt = _kind(q, "q")
    shape, kept = q.shape, k.shape
    if len(kept) != 4:
        raise ValueError(f"k and v must be [B, Lk, G, D] (got {tuple(kept)})")
    _, Lk, G, _ = kept
    if len(shape) == 4:
        B, Lq, H, D = shape
    else:
        (B, H, D), Lq = shape, 1
    kept = (B, Lk, G, D)
    if mask is None:
        mp, ms = None, 0
    else:
        if mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError(f"mask must be bool or uint8 (got {mask.dtype})")
        if mask.get_device() != q.get_device() or mask.shape != (B, Lk):
            _wrong(mask, mask.dtype, q.device, (B, Lk), "mask")
        mp, (ms, inner) = mask.data_ptr(), mask.stride()
        if inner != 1 and Lk > 1:
            raise ValueError("mask's last dimension must be dense")
    return CrossAttentionArgs(dt, B, Lq, Lk, H, G, D,
                              D ** -0.5 if scale is None else scale, _heads(q, q, shape, "q"), _heads(k, q, kept, "k"),
                              _heads(v, q, kept, "v"), _heads(y, q, shape, "y"), _i32(q_lengths, q, (B,), "q_lengths"),
                              _i32(lengths, q, (B,), "lengths"), mp, ms)


def _attention_ws(a, ref, which):
    return _scratch(_bytes("fdc_cross_attention_workspace_size", a.dtype, a.B, a.Lq, a.Lk, a.H, a.G, a.D, which=which, of=2),
                    ref)


def _saved_floats(a):
    return _bytes("fdc_cross_attention_saved_size", a.dtype, a.B, a.Lq, a.H, a.D) // 4


def cross_attention_forward(q, k, v, scale=None, q_lengths=None, lengths=None, mask=None, save=False, y=None):
    """Attention of q [B, Lq, H, D] to k and v [B, Lk, G, D], whose heads H / G adjacent ones of q share -> (y, saved)
    (fdc_cross_attention_forward).  scale: D ** -0.5 if None.  A sequence's keys are those before lengths [B] (int32) whose
    mask [B, Lk] (bool or uint8) is true, its queries those before q_lengths [B]; a row without keys is 0.
    saved (float32): what cross_attention_backward needs, if `save` is asked for, else None; its first B H Lq values are
    the logarithms of the rows' sums of exponentials, [B, H, Lq]."""
    if q.dim() != 4:
        raise ValueError(f"q must be [B, Lq, H, D] (got {tuple(q.shape)})")
    y = _like(q) if y is None else y
    a = _attention_args(q, k, v, scale, q_lengths, lengths, mask, y)
    saved = _empty((_saved_floats(a),), q, torch.float32) if save else None
    ws, size, keep = _attention_ws(a, q, 0)
    call("fdc_cross_attention_forward", a, _ptr(saved), ws, size, _stream())
    return y, saved


def cross_attention_step(q, k, v, scale=None, lengths=None, mask=None, y=None):
    """One token q [B, H, D] of every sequence -> y."""
    if q.dim() != 3:
        raise ValueError(f"q must be [B, H, D] (got {tuple(q.shape)})")
    y = _like(q) if y is None else y
    a = _attention_args(q, k, v, scale, None, lengths, mask, y)
    ws, size, keep = _attention_ws(a, q, 0)
    call("fdc_cross_attention_forward", a, None, ws, size, _stream())
    return y


def cross_attention_backward(gy, y, saved, q, k, v, scale=None, q_lengths=None, lengths=None, mask=None):
    """Gradients of q, k and v from gy and cross_attention_forward's y and what it saved."""
    if q.dim() != 4:
        raise ValueError(f"q must be [B, Lq, H, D] (got {tuple(q.shape)})")
    a = _attention_args(q, k, v, scale, q_lengths, lengths, mask, y)
    g = AttentionGradients(_like(q), _like(k), _like(v))
    s = CrossAttentionGrads(_heads(gy, q, q.shape, "gy"), _heads(g.q, q, q.shape, "gq"), _heads(g.k, q, k.shape, "gk"),
                            _heads(g.v, q, v.shape, "gv"))
    ws, size, keep = _attention_ws(a, q, 1)
    call("fdc_cross_attention_backward", a, _f32(saved, q, (_saved_floats(a),), "saved"), s, ws, size, _stream())
    return g


# ----------------------------------------------------------------------------
# token log probabilities
# ----------------------------------------------------------------------------
def _logprobs_args(z, tokens, K, temperature):
    dt = _kind(z, "z")
    if z.dim() != 2:
        raise ValueError(f"z must be [rows, vocabulary] (got {tuple(z.shape)})")
    return TokenLogprobsArgs(dt, z.shape[1], K, z.shape[0], temperature, *_rows(z, z, z.shape, "z"),
                             _i32(tokens, z, (z.shape[0],), "tokens"))


def token_logprobs_forward(z, tokens=None, top=0, temperature=1.0):
    """Of each row of z [rows, V] at a temperature (fdc_token_logprobs_forward): logp [rows], the log probability of
    tokens [rows] (int32, -1: none, which has 0; None without tokens), the entropy [rows], and the `top` best alternatives, idx
    [rows, top] (int32) and their log probabilities top [rows, top], from high to low, equal ones by place
    (None where top is 0) -> TokenLogprobs(logp, entropy, idx, top, stats)."""
    a = _logprobs_args(z, tokens, top, temperature)
    logp = None if tokens is None else _empty((a.R,), z, torch.float32)
    entropy, stats = _empty((a.R,), z, torch.float32), _empty((a.R, 3), z, torch.float32)
    idx, best = (_empty((a.R, top), z, torch.int32), _empty((a.R, top), z, torch.float32)) if top > 0 else (None, None)
    ws, size, keep = _scratch(_bytes("fdc_token_logprobs_workspace_size", a.dtype, a.R, a.V, a.K), z)
    call("fdc_token_logprobs_forward", a, _ptr(logp), _ptr(entropy), _ptr(idx), _ptr(best), _ptr(stats), ws, size, _stream())
    return TokenLogprobs(logp, entropy, idx, best, stats)


def token_logprobs_backward(stats, z, tokens=None, glogp=None, gentropy=None, idx=None, gtop=None, temperature=1.0,
                            gz=None):
    """Gradient of z from those of logp, entropy and top (None: 0; gtop with the forward's idx) and
    token_logprobs_forward's stats (gz may be z itself)."""
    if gtop is not None and (idx is None or idx.dim() != 2):
        raise ValueError("gtop goes with idx [rows, top]")
    K = 0 if gtop is None else idx.shape[1]
    a = _logprobs_args(z, tokens, K, temperature)
    gz = _like(z) if gz is None else gz
    gp, gs = _rows(gz, z, z.shape, "gz")
    named = (None, None) if gtop is None else (_i32(idx, z, (a.R, K), "idx"), _f32(gtop, z, (a.R, K), "gtop"))
    call("fdc_token_logprobs_backward", a, _f32(stats, z, (a.R, 3), "stats"), _f32(glogp, z, (a.R,), "glogp"),
         _f32(gentropy, z, (a.R,), "gentropy"), *named, gp, gs, _stream())
    return gz
