"""Outputs of the sequence operators that share memory with an input are refused before the GPU is touched, whatever
the strides' order; slices of one buffer that lie side by side are not.  (Each call that is not refused for its
activations is refused for its states, so that none reaches the GPU.)"""

import random

import pytest

from paper_2106_12736_amd import _lib
from paper_2106_12736_amd._lib import FDC_EINVAL, ConvArgs, DistillArgs, ScanArgs, Tokens

P = 0x100000  # never dereferenced: validation fails first


def _conv(x, y, B, L, D, n=4):
    # state and new_state half over each other
    a = ConvArgs(1, B, L, D, n, 1, x, y, P, None, P << 4, (P << 4) + 2, None)
    assert _lib.status("fdc_causal_conv_forward", a, None) == FDC_EINVAL
    return _lib.last_error()


def _elements(offset, B, L, D, bs, ts):
    return {offset + b * bs + t * ts + d for b in range(B) for t in range(L) for d in range(D)}


def test_conv_output_and_input():
    refused = accepted = 0
    rng = random.Random(1)
    for _ in range(4000):
        B, L, D = rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 5)
        gap, more = rng.randint(0, 7), rng.randint(0, 9)
        if rng.random() < 0.5:
            ts, bs = D + gap, L * (D + gap) + more
        else:
            bs, ts = D + gap, B * (D + gap) + more
        shift = rng.randint(-2 * B * L * D, 2 * B * L * D)
        over = bool(_elements(0, B, L, D, bs, ts) & _elements(shift, B, L, D, bs, ts))
        same_token = shift == 0 and L == 1  # y may be x there
        said = _conv(Tokens(P, bs, ts), Tokens(P + 2 * shift, bs, ts), B, L, D)
        expected = "y shares memory with x" if over and not same_token else "new_state and state share memory in part"
        assert said == expected, (B, L, D, bs, ts, shift, said)
        refused, accepted = refused + (said[0] == "y"), accepted + (said[0] == "n")
    assert refused > 500 and accepted > 500


def test_conv_same_address_other_strides():
    assert _conv(Tokens(P, 0, 0), Tokens(P, 48, 8), 2, 6, 8) == "y shares memory with x"


def test_conv_backward():
    t = Tokens(P, 48, 8)
    other, apart = Tokens(P << 1, 48, 8), Tokens(P << 2, 48, 8)
    for x, gy, gx, name in ((t, other, t, "x"), (t, other, other, "gy"), (t, other, Tokens(P + 16, 48, 8), "x"),
                            (apart, other, Tokens((P << 1) - 2, 48, 8), "gy")):
        a = ConvArgs(1, 2, 6, 8, 4, 1, x, t, P, None, None, None, None)
        assert _lib.status("fdc_causal_conv_backward", a, gy, gx, None, None, None, 0, None) == FDC_EINVAL
        assert _lib.last_error() == f"gx shares memory with {name}"


@pytest.mark.parametrize("name,entry", [("fdc_scan_forward", (None, None, 0, None)), ("fdc_scan_step", (None,))])
def test_scan(name, entry):
    B, L, D, N = 2, 1 if "step" in name else 6, 8, 4

    def say(**change):
        at = {k: Tokens(P * (i + 1), 240, 40) for i, k in enumerate(("x", "dt", "gate", "Bm", "Cm", "y"))}
        at.update(change)
        a = ScanArgs(1, B, L, D, N, 2, 1, *at.values(), P, None, None, P << 8, (P << 8) + 16, None)
        assert _lib.status(name, a, *entry) == FDC_EINVAL
        return _lib.last_error()

    fine = "h_last and h0 share memory in part"
    assert say() == fine
    for i, k in enumerate(("x", "dt", "gate", "Bm", "Cm")):
        whole, side, part = (Tokens(P * (i + 1) + s, 240, 40) for s in (0, 16, 14))
        assert say(y=whole) == (fine if i < 3 else f"y shares memory with {k}")
        assert say(y=side) == fine
        assert say(y=part) == f"y shares memory with {k}"


def test_distill_gradient_over_logits():
    a = DistillArgs(1, 8, 2, 5, 1.0, 0.5, P, 16, P, P, P, P)
    for gz, stride in ((P + 2, 16), (P + 32, 16), (P - 96, 16), (P - 14, 16), (P, 17)):
        assert _lib.status("fdc_distill_backward", a, P, P, gz, stride, None) == FDC_EINVAL
        assert _lib.last_error() == "gz shares memory with z"
        assert _lib.status("fdc_distill_forward_backward", a, P, P, P, gz, stride, P, 1 << 40, None) == FDC_EINVAL
        assert _lib.last_error() == "gz shares memory with z"
