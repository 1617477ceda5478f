"""The sequence operators together: the example's student learns from its teacher, its gradients are those
of its loss, and its answers token by token are those of the whole pass."""

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _parts():
    import sequence_student as ex

    tokens = ex.features()[:4, :200].contiguous()
    return ex, tokens, ex.teach(tokens, codes=128, K=8, teacher_inner=64)


def test_student_learns():
    ex, tokens, taught = _parts()
    student = ex.Network(tokens.shape[-1], 48, 16, 4, 2, 128, seed=2)
    losses = ex.train(student, tokens, *taught, steps=25)
    print(losses, flush=True)
    # a student that learnt nothing stays where it starts
    assert losses[-1] < 0.7 * losses[0]


def test_gradient_along_itself():
    # the loss along the gradient: central differences over a step that changes it by some percent, in bf16
    # activations (2^-8 each, averaged over 800 tokens), so 5 percent
    ex, tokens, (idx, logits, labels) = _parts()
    student = ex.Network(tokens.shape[-1], 48, 16, 4, 2, 128, seed=3)
    rows = idx.shape[0]
    up = torch.full((rows,), 1.0 / rows, device="cuda")

    def loss():
        z, kept, _ = student.forward(tokens)
        out, gz = ex.seq.distill_forward_backward(up, z, idx, logits, temperature=2.0, labels=labels, alpha=0.7)
        return out.double().mean(), gz, kept

    mean, gz, kept = loss()
    student.backward(gz, kept, tokens.shape)
    g = student.grad.clone()
    square = float((g.double() ** 2).sum())
    eps = 0.05 * float(mean) / square
    start = student.flat.clone()
    ends = []
    for s in (eps, -eps):
        student.flat.copy_(start + s * g)
        ends.append(float(loss()[0]))
    slope = (ends[0] - ends[1]) / (2 * eps)
    print(slope, square, flush=True)
    assert abs(slope - square) <= 0.05 * square


def test_token_by_token():
    ex, tokens, taught = _parts()
    student = ex.Network(tokens.shape[-1], 48, 16, 4, 2, 128, seed=4)
    whole = student.forward(tokens)[0].view(*tokens.shape[:2], -1)
    _, _, states = student.forward(tokens[:, :150].contiguous(), last=True)
    for t in range(150, 200):
        z = student.step(tokens[:, t].contiguous(), states).float()
        want = whole[:, t].float()
        # about ten roundings to bf16 one after another on either side, at most 2^-8 each
        assert float((z - want).norm() / want.norm()) <= 10 * 2.0 ** -8, t
