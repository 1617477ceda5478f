"""A small sequence network on an FDCNN's features, taught by a larger one's top logits, then run token by token.

The FDCNN chain's output planes [B][C][M][M] are read as M * M tokens of C channels.  Teacher and student
are the same kind of network over them: blocks of a causal convolution and a selective state space scan
between the norms, gate and residual scale of `block_norm`, then a projection to codes.  Of the teacher
only its K best logits a token are kept; the student is trained on them with Adam (fdc_adam_step), and
then answers one token at a time from the states its blocks carry.

    python examples/sequence_student.py [--steps 30]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2106_12736_amd import inputs, layers, sequence as seq  # noqa: E402
from paper_2106_12736_amd._lib import call  # noqa: E402

T = torch.bfloat16


def _mm(a, b):
    """A plain product over the last dimension of a, with its rows side by side."""
    return (a.reshape(-1, a.shape[-1]) @ b).view(*a.shape[:-1], b.shape[-1])


def _wgrad(a, g):
    return (a.reshape(-1, a.shape[-1]).t().contiguous() @ g.reshape(-1, g.shape[-1])).float()


class Network:
    """`depth` blocks of `inner` channels on tokens of D, and a projection to V codes.  All parameters are
    views of one float32 buffer, their gradients of another, so that one launch updates them."""

    def __init__(self, D, inner, states, taps, depth, V, seed, device="cuda"):
        self.D, self.inner, self.states, self.taps, self.depth = D, inner, states, taps, depth
        shapes = {"w_in": (D, 3 * inner + 2 * states), "conv_w": (inner, taps), "conv_b": (inner,), "A_log": (inner, states),
                  "skip": (inner,), "dt_bias": (inner,), "w_out": (inner, D), "scale": (D,), "w_post": (D,), "w_pre": (D,)}
        names = [("first", (D,))] + [(f"{k}.{i}", s) for i in range(depth) for k, s in shapes.items()] + [("head", (D, V))]
        sizes = [torch.Size(s).numel() for _, s in names]
        self.flat = torch.empty(sum(sizes), device=device)
        self.grad, self.m, self.v = (torch.zeros_like(self.flat) for _ in range(3))
        self.count = torch.zeros(1, dtype=torch.int32, device=device)
        cut = lambda buf: {n: t.view(s) for (n, s), t in zip(names, buf.split(sizes))}  # noqa: E731
        self.p, self.g = cut(self.flat), cut(self.grad)
        gen = torch.Generator(device=device).manual_seed(seed)
        start = {"conv_b": 0.0, "skip": 1.0, "scale": 0.5, "w_post": 1.0, "w_pre": 1.0, "first": 1.0, "dt_bias": -3.0}
        for n, t in self.p.items():
            kind = n.split(".")[0]
            if kind == "A_log":
                t.copy_(torch.arange(1, states + 1, device=device).float().log())
            elif kind in start:
                t.fill_(start[kind])
            else:
                t.normal_(generator=gen).mul_((taps if kind == "conv_w" else t.shape[0]) ** -0.5)

    def _block(self, i):
        return {k.split(".")[0]: t for k, t in self.p.items() if k.endswith(f".{i}")}

    def _split(self, p):
        """x, gate, dt, B and C of a block's input projection, where they lie."""
        c, n = self.inner, self.states
        return (p[..., :c], p[..., c:2 * c], p[..., 2 * c:3 * c], p[..., None, 3 * c:3 * c + n], p[..., None, 3 * c + n:])

    def forward(self, tokens, last=False):
        """Logits of [B, L, D] tokens (bf16), what the backward needs, and the states after the last token."""
        B, L, D = tokens.shape
        x = tokens.reshape(-1, D)
        _, n, stats0 = seq.block_norm_forward(x, w_pre=self.p["first"])
        kept, states = [(x, stats0)], []
        for i in range(self.depth):
            b = self._block(i)
            A = -torch.exp(b["A_log"])
            proj = _mm(n.view(B, L, D), b["w_in"].to(T))
            xs, gate, dt, Bm, Cm = self._split(proj)
            c, tail = seq.causal_conv_forward(xs, b["conv_w"], bias=b["conv_b"], silu=True, last=last)
            y, h, saved = seq.scan_forward(c, dt, A, Bm, Cm, skip=b["skip"], gate=gate, dt_bias=b["dt_bias"], last=last,
                                           save=True)
            f = _mm(y, b["w_out"].to(T)).view(-1, D)
            out, after, stats = seq.block_norm_forward(x, f, scale=b["scale"], w_post=b["w_post"], w_pre=b["w_pre"])
            kept.append((n, proj, c, A, saved, y, x, f, stats))
            states.append((tail, h))
            x, n = out, after
        kept.append(n)
        return _mm(n, self.p["head"].to(T)), kept, states

    def backward(self, gz, kept, shape):
        B, L, D = shape
        n = kept[-1]
        self.g["head"].copy_(_wgrad(n, gz))
        gn, gout = gz @ self.p["head"].to(T).t().contiguous(), None
        for i in reversed(range(self.depth)):
            b, g = self._block(i), {k.split(".")[0]: t for k, t in self.g.items() if k.endswith(f".{i}")}
            n, proj, c, A, saved, y, x, f, stats = kept[i + 1]
            r = seq.block_norm_backward(gout, gn, stats, x, f, scale=b["scale"], w_post=b["w_post"], w_pre=b["w_pre"])
            g["scale"].copy_(r.scale), g["w_post"].copy_(r.w_post), g["w_pre"].copy_(r.w_pre)
            gout, gf = r.x, r.f
            g["w_out"].copy_(_wgrad(y, gf))
            gy = _mm(gf.view(B, L, D), b["w_out"].to(T).t().contiguous())
            xs, gate, dt, Bm, Cm = self._split(proj)
            s = seq.scan_backward(gy, saved, c, dt, A, Bm, Cm, skip=b["skip"], gate=gate, dt_bias=b["dt_bias"])
            g["A_log"].copy_(s.A * A), g["skip"].copy_(s.skip), g["dt_bias"].copy_(s.dt_bias)
            gxs, gw, gbias = seq.causal_conv_backward(s.x, xs, b["conv_w"], bias=b["conv_b"], silu=True)
            g["conv_w"].copy_(gw), g["conv_b"].copy_(gbias)
            gproj = torch.cat([gxs, s.gate, s.dt, s.B.squeeze(-2), s.C.squeeze(-2)], -1).view(B * L, -1)
            g["w_in"].copy_(_wgrad(n, gproj))
            gn = gproj @ b["w_in"].to(T).t().contiguous()
        x, stats0 = kept[0]
        self.g["first"].copy_(seq.block_norm_backward(gout, gn, stats0, x, w_pre=self.p["first"]).w_pre)

    def adam(self, lr):
        ptr = [t.data_ptr() for t in (self.flat, self.grad, self.m, self.v)]
        call("fdc_adam_step", *ptr, self.flat.numel(), self.count.data_ptr(), lr, 0.9, 0.999, 1e-8, 0.0, layers._stream())

    def step(self, token, states):
        """Logits of one token [B, D] of every sequence; the blocks' states are updated in place."""
        x = token
        _, n, _ = seq.block_norm_forward(x, w_pre=self.p["first"])
        for i, (tail, h) in enumerate(states):
            b = self._block(i)
            xs, gate, dt, Bm, Cm = self._split(n @ b["w_in"].to(T))
            c, _ = seq.causal_conv_step(xs, b["conv_w"], tail, bias=b["conv_b"], silu=True)
            y, _ = seq.scan_step(c, dt, -torch.exp(b["A_log"]), Bm, Cm, h, skip=b["skip"], gate=gate, dt_bias=b["dt_bias"])
            x, n, _ = seq.block_norm_forward(x, y @ b["w_out"].to(T), scale=b["scale"], w_post=b["w_post"],
                                             w_pre=b["w_pre"])
        return n @ self.p["head"].to(T)


def features(wl=inputs.STACK256, device="cuda"):
    """Tokens [B, M * M, C] of the FDCNN chain's output, of unit size."""
    d = inputs.make_cic_stack(wl)
    chain = layers.CicChain(wl.batch, wl.sizes, wl.channels, device=device)
    out = chain.forward(torch.from_numpy(d.x).to(device), [torch.from_numpy(k).to(device) for k in d.kernels])
    tokens = out.flatten(2).transpose(1, 2)
    return (tokens / tokens.std()).to(T).contiguous()


def teach(tokens, codes, K, teacher_inner=256):
    """The teacher's K best logits of every token, their places and the best one as a label."""
    teacher = Network(tokens.shape[-1], teacher_inner, 16, 4, 2, codes, seed=1)
    top = (teacher.forward(tokens)[0].float() * 4).topk(K, dim=-1)
    idx = top.indices.to(torch.int32).view(-1, K)
    return idx, top.values.to(T).view(-1, K), idx[:, 0].contiguous()


def train(student, tokens, idx, logits, labels, steps, lr=2e-3, temperature=2.0, alpha=0.7):
    """Mean loss of every step."""
    rows = idx.shape[0]
    up = torch.full((rows,), 1.0 / rows, device=tokens.device)
    losses = []
    for _ in range(steps):
        z, kept, _ = student.forward(tokens)
        loss, gz = seq.distill_forward_backward(up, z, idx, logits, temperature=temperature, labels=labels, alpha=alpha)
        student.backward(gz, kept, tokens.shape)
        student.adam(lr)
        losses.append(loss.mean())
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    tokens = features()
    idx, logits, labels = teach(tokens, codes=512, K=16)
    student = Network(tokens.shape[-1], 64, 16, 4, 2, 512, seed=2)
    losses = train(student, tokens, idx, logits, labels, a.steps)
    for i in range(0, a.steps, max(1, a.steps // 6)):
        print(f"step {i}: loss {losses[i]:.4f}", flush=True)
    print(f"step {a.steps - 1}: loss {losses[-1]:.4f}", flush=True)

    # a prompt in one pass, then token by token
    whole = student.forward(tokens)[0]
    prompt = tokens.shape[1] - 16
    _, _, states = student.forward(tokens[:, :prompt].contiguous(), last=True)
    worst = 0.0
    for t in range(prompt, tokens.shape[1]):
        z = student.step(tokens[:, t].contiguous(), states)
        want = whole.view(*tokens.shape[:2], -1)[:, t].float()
        worst = max(worst, float((z.float() - want).norm() / want.norm()))
    print(f"token by token: logits within {worst:.1e} of the whole pass's")


if __name__ == "__main__":
    main()
