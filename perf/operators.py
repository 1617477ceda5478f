"""What the speed of the sequence operators is measured on: the calls that a user's program makes
through `paper_2106_12736_amd.sequence`, over the sizes that such programs have.

A sequence network takes tokens where an FDCNN takes images (or the pixels of an FDCNN's last planes
as tokens).  Its block is a short causal convolution, a selective state space scan and the norms,
gate and residual scale around them; it is trained with a loss against a teacher's top logits.

  conv     causal convolution of each channel with its own short kernel: `train` (forward and
           backward), `step` (one token, with the state of the last tokens)
  scan     selective state space scan: `train`, `prompt` (forward, the last state kept), `step`
  norm     norm of a block's output, gate, residual scale and the norm before the next block:
           `train`, `serve` (forward alone)
  distill  the loss against a teacher's top logits: `train` (loss and gradient in one call), `split`
           (loss, then the gradient from an upstream one)

Activations are bf16, f16 or f32; parameters and states are f32.
"""

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def listed():
    return [
        # one sequence being answered token by token: launches and latency
        {"name": "conv_step_b1", "op": "conv", "mode": "step", "B": 1, "L": 1, "D": 2048, "n": 4, "dtype": "bf16",
         "ragged": False},
        # a training step's convolution at a full batch
        {"name": "conv_train_b8_l2048", "op": "conv", "mode": "train", "B": 8, "L": 2048, "D": 4096, "n": 4,
         "dtype": "bf16", "ragged": False},
        # sequences of unlike lengths (one of them empty) that go on from earlier tokens, odd channels, f32
        {"name": "conv_ragged_f32", "op": "conv", "mode": "train", "B": 3, "L": 777, "D": 1030, "n": 3,
         "dtype": "f32", "ragged": True},
        # 64 sequences answered together
        {"name": "scan_step_b64", "op": "scan", "mode": "step", "B": 64, "L": 1, "D": 4096, "N": 16, "G": 1,
         "dtype": "f16", "ragged": False},
        # one long prompt: few channels, so the work has to come from along the sequence
        {"name": "scan_prompt_l16384", "op": "scan", "mode": "prompt", "B": 1, "L": 16384, "D": 2048, "N": 16,
         "G": 1, "dtype": "bf16", "ragged": False},
        # a training step over the 32 x 32 pixels of a stack's last planes as tokens, the stack's batch of 8
        {"name": "scan_train_b8_l1024", "op": "scan", "mode": "train", "B": 8, "L": 1024, "D": 2048, "N": 16,
         "G": 1, "dtype": "bf16", "ragged": False},
        # unlike lengths, two groups of channels, a state and a width that fill no tile, f32
        {"name": "scan_ragged_f32", "op": "scan", "mode": "train", "B": 3, "L": 509, "D": 330, "N": 10, "G": 2,
         "dtype": "f32", "ragged": True},
        # the norms of one token of 8 sequences
        {"name": "norm_serve_r8", "op": "norm", "mode": "serve", "R": 8, "D": 4096, "act": "silu", "dtype": "f16"},
        # a training step's norms at a full batch
        {"name": "norm_train_r16384", "op": "norm", "mode": "train", "R": 16384, "D": 2048, "act": "silu",
         "dtype": "bf16"},
        # an odd width and number of tokens in f32
        {"name": "norm_odd_f32", "op": "norm", "mode": "train", "R": 1001, "D": 777, "act": "sigmoid",
         "dtype": "f32"},
        # the loss of a training step: 4096 tokens over a large vocabulary, the teacher's 64 best kept
        {"name": "distill_train_r4096", "op": "distill", "mode": "train", "R": 4096, "V": 32000, "K": 64,
         "dtype": "bf16"},
        # a few answers over an odd vocabulary, some tokens without a teacher, label or weight
        {"name": "distill_split_r7", "op": "distill", "mode": "split", "R": 7, "V": 50021, "K": 10, "dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(["conv", "scan", "scan", "norm", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "conv":
        mode = rng.choice(["train", "train", "step"])
        return {"op": op, "mode": mode, "B": _log_int(rng, 1, 256 if mode == "step" else 16),
                "L": 1 if mode == "step" else _log_int(rng, 2, 8192), "D": _log_int(rng, 64, 8192),
                "n": rng.choice([2, 3, 4, 4]), "dtype": dtype, "ragged": mode == "train" and rng.random() < 0.3}
    if op == "scan":
        mode = rng.choice(["train", "train", "prompt", "step"])
        G = rng.choice([1, 1, 1, 2, 4])
        return {"op": op, "mode": mode, "B": _log_int(rng, 1, 256 if mode == "step" else 16),
                "L": 1 if mode == "step" else _log_int(rng, 2, 4096 if mode == "train" else 16384),
                "D": G * _log_int(rng, 16, 4096 // G), "N": rng.choice([16, 16, 16, 8, 32, rng.randint(1, 64)]),
                "G": G, "dtype": dtype, "ragged": mode != "step" and rng.random() < 0.3}
    if op == "norm":
        mode = rng.choice(["train", "serve"])
        return {"op": op, "mode": mode, "R": _log_int(rng, 1, 32768), "D": _log_int(rng, 64, 8192),
                "act": rng.choice(["silu", "sigmoid"]), "dtype": dtype}
    V = _log_int(rng, 100, 200000)
    return {"op": op, "mode": rng.choice(["train", "split"]), "R": _log_int(rng, 1, 8192), "V": V,
            "K": _log_int(rng, 1, 96), "dtype": dtype}


def _cost(case):
    """A rough count of a pass's work, to keep drawn cases within the listed ones."""
    if case["op"] == "scan" and case["mode"] != "step":
        return case["B"] * case["L"] * case["D"] * case["N"] * (3 if case["mode"] == "train" else 1)
    return work(case)["bytes"]


def draw(rng):
    most = {}
    for c in listed():
        kind = "pass" if c["op"] == "scan" and c["mode"] != "step" else "bytes"
        most[kind] = max(most.get(kind, 0), _cost(c))
    while True:
        c = _draw_once(rng)
        kind = "pass" if c["op"] == "scan" and c["mode"] != "step" else "bytes"
        if _cost(c) <= most[kind]:
            return c


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------
def _lengths(case, g):
    """Unlike lengths from 0 to L: the first sequence is whole and the last one empty (where there are several)."""
    B, L = case["B"], case["L"]
    n = torch.randint(0, L + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    n[-1] = 0
    n[0] = L
    return n


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    T = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, mean=0.0):
        return torch.randn(shape, generator=g, device=DEV) * scale + mean

    s = {"op": case["op"], "mode": case["mode"], "lengths": None}
    if case["op"] == "conv":
        B, L, D, n = case["B"], case["L"], case["D"], case["n"]
        shape = (B, D) if case["mode"] == "step" else (B, L, D)
        s.update(x=normal(*shape).to(T), w=normal(D, n, scale=n ** -0.5), bias=normal(D, scale=0.1), silu=True,
                 state=None)
        if case["mode"] == "step" or case["ragged"]:
            s["state"] = normal(B, n - 1, D).to(T)
        if case["ragged"]:
            s["lengths"] = _lengths(case, g)
        if case["mode"] == "train":
            s["gy"] = normal(B, L, D).to(T)
        return s
    if case["op"] == "scan":
        B, L, D, N, G = case["B"], case["L"], case["D"], case["N"], case["G"]
        lead = (B,) if case["mode"] == "step" else (B, L)
        # the usual start of such a layer: A = -1 .. -N in every channel (here as it is after some training), step
        # sizes spread over 0.001 .. 0.1 by their bias
        A = -torch.arange(1, N + 1, device=DEV, dtype=torch.float32) * torch.exp(normal(D, N, scale=0.1))
        rate = torch.exp(torch.rand((D,), generator=g, device=DEV) * (math.log(0.1) - math.log(0.001)) +
                         math.log(0.001))
        s.update(x=normal(*lead, D).to(T), dt=normal(*lead, D, scale=0.5).to(T), A=A,
                 B=normal(*lead, G, N).to(T), C=normal(*lead, G, N).to(T), skip=normal(D, scale=0.1, mean=1.0),
                 gate=normal(*lead, D).to(T), dt_bias=torch.log(torch.expm1(rate)), h0=None)
        if case["mode"] == "step" or case["ragged"]:
            s["h0"] = normal(B, D, N, scale=0.1)
        if case["ragged"]:
            s["lengths"] = _lengths(case, g)
        if case["mode"] == "train":
            s["gy"] = normal(B, L, D).to(T)
        return s
    if case["op"] == "norm":
        R, D = case["R"], case["D"]
        s.update(x=normal(R, D, scale=2.0).to(T), f=normal(R, D).to(T), gate=normal(R, D).to(T),
                 scale=normal(D, scale=0.02, mean=0.1), w_post=normal(D, scale=0.1, mean=1.0),
                 w_pre=normal(D, scale=0.1, mean=1.0), act=case["act"])
        if case["mode"] == "train":
            s.update(gout=normal(R, D).to(T), gn=normal(R, D).to(T))
        return s
    R, V, K = case["R"], case["V"], min(case["K"], case["V"])
    z = normal(R, V, scale=2.0).to(T)
    # the teacher agrees with the student in part; what is kept of it are its K best logits, from high to low
    top = (z.float() * 0.7).add_(normal(R, V, scale=1.5)).topk(K, dim=1)
    idx, teacher = top.indices.to(torch.int32), top.values.to(T)
    labels = idx[:, 0].clone()
    weight = torch.ones(R, device=DEV)
    if case["mode"] == "split":  # padding and other tokens that have no label, teacher or weight
        u = torch.rand((R, 3), generator=g, device=DEV)
        labels[u[:, 0] < 0.2] = -1
        idx[u[:, 1] < 0.2] = -1
        idx[:, K // 2 + 1:][(u[:, 1] > 0.7)] = -1
        weight[u[:, 2] < 0.2] = 0.0
    s.update(z=z, idx=idx, teacher=teacher, labels=labels, weight=weight, temperature=2.0, alpha=0.75,
             gloss=torch.full((R,), 1.0 / R, device=DEV) * (1 + 0.1 * normal(R)))
    return s


# ----------------------------------------------------------------------------
# the passes: the framework's calls
# ----------------------------------------------------------------------------
def _own_conv(s):
    from paper_2106_12736_amd import sequence as seq

    if s["mode"] == "step":
        y, state = seq.causal_conv_step(s["x"], s["w"], s["state"], bias=s["bias"], silu=s["silu"],
                                        new_state=torch.empty_like(s["state"]))
        return {"y": y, "state": state}
    y, state = seq.causal_conv_forward(s["x"], s["w"], bias=s["bias"], silu=s["silu"], state=s["state"],
                                       lengths=s["lengths"], last=True)
    gx, gw, gbias = seq.causal_conv_backward(s["gy"], s["x"], s["w"], bias=s["bias"], silu=s["silu"],
                                             state=s["state"], lengths=s["lengths"])
    return {"y": y, "state": state, "gx": gx, "gw": gw, "gbias": gbias}


def _own_scan(s):
    from paper_2106_12736_amd import sequence as seq

    kw = {"skip": s["skip"], "gate": s["gate"], "dt_bias": s["dt_bias"]}
    if s["mode"] == "step":
        y, h = seq.scan_step(s["x"], s["dt"], s["A"], s["B"], s["C"], s["h0"], h_new=torch.empty_like(s["h0"]), **kw)
        return {"y": y, "h": h}
    train = s["mode"] == "train"
    y, h, saved = seq.scan_forward(s["x"], s["dt"], s["A"], s["B"], s["C"], h0=s["h0"], lengths=s["lengths"],
                                   last=True, save=train, **kw)
    if not train:
        return {"y": y, "h": h}
    g = seq.scan_backward(s["gy"], saved, s["x"], s["dt"], s["A"], s["B"], s["C"], lengths=s["lengths"], **kw)
    return {"y": y, "h": h, "gx": g.x, "gdt": g.dt, "gA": g.A, "gB": g.B, "gC": g.C, "gskip": g.skip,
            "ggate": g.gate, "gdt_bias": g.dt_bias}


def _own_norm(s):
    from paper_2106_12736_amd import sequence as seq

    kw = {"scale": s["scale"], "w_post": s["w_post"], "w_pre": s["w_pre"], "act": s["act"], "eps": EPS}
    out, n, stats = seq.block_norm_forward(s["x"], s["f"], s["gate"], **kw)
    if s["mode"] == "serve":
        return {"out": out, "n": n}
    g = seq.block_norm_backward(s["gout"], s["gn"], stats, s["x"], s["f"], s["gate"], **kw)
    return {"out": out, "n": n, "gx": g.x, "gf": g.f, "ggate": g.gate, "gscale": g.scale, "gw_post": g.w_post,
            "gw_pre": g.w_pre}


def _own_distill(s):
    from paper_2106_12736_amd import sequence as seq

    kw = {"temperature": s["temperature"], "labels": s["labels"], "alpha": s["alpha"], "weight": s["weight"]}
    if s["mode"] == "train":
        loss, gz = seq.distill_forward_backward(s["gloss"], s["z"], s["idx"], s["teacher"], **kw)
    else:
        loss, stats = seq.distill_forward(s["z"], s["idx"], s["teacher"], **kw)
        gz = seq.distill_backward(s["gloss"], stats, s["z"], s["idx"], s["teacher"], **kw)
    return {"loss": loss, "gz": gz}


# ----------------------------------------------------------------------------
# the passes: plain forms
# ----------------------------------------------------------------------------
def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _live(lengths, shape, like):
    """[B][L] truth values: whether a token lies within its sequence."""
    t = torch.arange(shape[1], device=like.device)
    if lengths is None:
        return torch.ones(shape[:2], dtype=torch.bool, device=like.device)
    return t[None, :] < lengths[:, None]


def _plain_conv(s):
    T, w, n = s["x"].dtype, s["w"], s["w"].shape[1]
    step = s["mode"] == "step"
    x = (s["x"][:, None] if step else s["x"]).float()
    B, L, D = x.shape
    past = s["state"].float() if s["state"] is not None else x.new_zeros(B, n - 1, D)
    live = _live(s["lengths"], x.shape, x)[..., None]
    x = torch.where(live, x, 0.0)
    xp = torch.cat([past, x], 1)
    taps = xp.unfold(1, n, 1)  # [B][L][D][n]
    p = (taps * w).sum(-1) + s["bias"]
    sg = _sigmoid(p)
    y = torch.where(live, p * sg, 0.0)
    count = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), L, device=x.device)
    rows = (count[:, None] + torch.arange(n - 1, device=x.device))[..., None].expand(B, n - 1, D)
    state = xp.gather(1, rows).to(T)
    if step:
        return {"y": y[:, 0].to(T), "state": state}
    gp = torch.where(live, s["gy"].float() * (sg * (1.0 + p * (1.0 - sg))), 0.0)
    gpp = torch.cat([gp, gp.new_zeros(B, n - 1, D)], 1)
    gx = torch.where(live, (gpp.unfold(1, n, 1) * w.flip(1)).sum(-1), 0.0)
    return {"y": y.to(T), "state": state, "gx": gx.to(T), "gw": (gp[..., None] * taps).sum((0, 1)),
            "gbias": gp.sum((0, 1))}


def _recur(a, b):
    """h[t] = a[t] h[t-1] + b[t] along dimension 1 (h[-1] = 0), by doubling the span that a value covers."""
    span = 1
    while span < a.shape[1]:
        b = torch.cat([b[:, :span], torch.addcmul(b[:, span:], a[:, span:], b[:, :-span])], 1)
        a = torch.cat([a[:, :span], a[:, span:] * a[:, :-span]], 1)
        span *= 2
    return b


def _plain_scan(s):
    T, A = s["x"].dtype, s["A"]
    step = s["mode"] == "step"
    x, dt, Bm, Cm, gate = ((s[k][:, None] if step else s[k]).float() for k in ("x", "dt", "B", "C", "gate"))
    L, D = x.shape[1:]
    live = _live(s["lengths"], x.shape, x)[..., None]
    raw = dt + s["dt_bias"]
    delta = torch.where(live, raw.clamp(min=0) + torch.log1p(torch.exp(-raw.abs())), 0.0)
    x = torch.where(live, x, 0.0)
    per = D // Bm.shape[2]
    Bd, Cd = (v.repeat_interleave(per, 2) for v in (Bm, Cm))  # [B][L][D][N]
    a = torch.exp(delta[..., None] * A)
    b = (delta * x)[..., None] * Bd
    if s["h0"] is not None:
        b[:, 0] += a[:, 0] * s["h0"]
    h = _recur(a, b)
    scanned = (h * Cd).sum(-1) + s["skip"] * x
    sg = _sigmoid(gate)
    y = torch.where(live, scanned * gate * sg, 0.0)
    if step:
        return {"y": y[:, 0].to(T), "h": h[:, 0]}
    out = {"y": y.to(T), "h": h[:, -1].clone()}
    if s["mode"] == "prompt":
        return out
    gy = torch.where(live, s["gy"].float(), 0.0)
    gs = gy * gate * sg
    # adjoint of the states, from the last token to the first: g[t] = a[t+1] g[t+1] + C[t] gs[t]
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    gh = _recur(after.flip(1), (gs[..., None] * Cd).flip(1)).flip(1)
    first = s["h0"][:, None] if s["h0"] is not None else torch.zeros_like(h[:, :1])
    before = torch.cat([first, h[:, :-1]], 1)
    gexp = gh * before * a  # gradient of delta A
    gu = (gh * Bd).sum(-1)  # gradient of delta x
    gdelta = (gexp * A).sum(-1) + gu * x
    graw = torch.where(live, gdelta * _sigmoid(raw), 0.0)
    shape = Bm.shape[:3] + (per, Bm.shape[3])
    live4 = live[..., None]
    gB = torch.where(live4, (gh * (delta * x)[..., None]).view(shape).sum(3), 0.0)
    gC = torch.where(live4, (h * gs[..., None]).view(shape).sum(3), 0.0)
    gx = torch.where(live, gu * delta + gs * s["skip"], 0.0)
    ggate = gy * scanned * sg * (1.0 + gate * (1.0 - sg))
    out.update(gx=gx.to(T), gdt=graw.to(T), gA=(gexp * delta[..., None]).sum((0, 1)), gB=gB.to(T), gC=gC.to(T),
               gskip=(gs * x).sum((0, 1)), ggate=torch.where(live, ggate, 0.0).to(T), gdt_bias=graw.sum((0, 1)))
    return out


def _plain_norm(s):
    T = s["x"].dtype
    x, f, gate = (s[k].float() for k in ("x", "f", "gate"))
    sg = _sigmoid(gate)
    act = gate * sg if s["act"] == "silu" else sg
    rf = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    post = f * rf * s["w_post"]
    out = x + s["scale"] * act * post
    ro = torch.rsqrt((out * out).mean(-1, keepdim=True) + EPS)
    n = out * ro * s["w_pre"]
    got = {"out": out.to(T), "n": n.to(T)}
    if s["mode"] == "serve":
        return got
    gn = s["gn"].float()
    v = gn * s["w_pre"]
    go = s["gout"].float() + v * ro - out * ro ** 3 * (v * out).mean(-1, keepdim=True)
    gpost = go * s["scale"] * act
    u = gpost * s["w_post"]
    slope = sg * (1.0 + gate * (1.0 - sg)) if s["act"] == "silu" else sg * (1.0 - sg)
    got.update(gx=go.to(T), gf=(u * rf - f * rf ** 3 * (u * f).mean(-1, keepdim=True)).to(T),
               ggate=(go * s["scale"] * post * slope).to(T), gscale=(go * act * post).sum(0),
               gw_post=(gpost * f * rf).sum(0), gw_pre=(gn * out * ro).sum(0))
    return got


def _softmax(z, m):
    """Softmax of rows whose largest value is m, and the logarithm of the sum of their exponentials."""
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    return e / total, m + torch.log(total)


def _plain_distill(s):
    z, tau, alpha = s["z"].float(), s["temperature"], s["alpha"]
    has, labelled = s["idx"] >= 0, (s["labels"] >= 0)[:, None]
    at = s["idx"].long().clamp(min=0)
    taught = has.any(1, keepdim=True)
    t = torch.where(has, s["teacher"].float() / tau, float("-inf"))
    best = torch.where(taught, t.amax(1, keepdim=True), 0.0)
    e = torch.exp(t - best)
    total = torch.where(taught, e.sum(1, keepdim=True), 1.0)
    q = e / total
    m = z.amax(1, keepdim=True)
    p1, lse1 = _softmax(z, m)
    pt, lset = _softmax(z / tau, m / tau)
    kl = torch.where(has, q * ((t - best - torch.log(total)) - (z.gather(1, at) / tau - lset)), 0.0)
    label = s["labels"].long().clamp(min=0)[:, None]
    hard = torch.where(labelled, lse1 - z.gather(1, label), 0.0)
    loss = s["weight"] * ((1 - alpha) * hard[:, 0] + alpha * tau * tau * kl.sum(1))
    gz = (1 - alpha) * labelled * p1 + alpha * tau * taught * pt
    gz.scatter_add_(1, at, -alpha * tau * q)
    gz.scatter_add_(1, label, -(1 - alpha) * labelled.float())
    return {"loss": loss, "gz": (gz * (s["gloss"] * s["weight"])[:, None]).to(s["z"].dtype)}


OWN = {"conv": _own_conv, "scan": _own_scan, "norm": _own_norm, "distill": _own_distill}
PLAIN = {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm, "distill": _plain_distill}


def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    e, mode = SIZE[case["dtype"]], case["mode"]
    if case["op"] == "conv":
        B, L, D, n = case["B"], case["L"], case["D"], case["n"]
        past = e * B * (n - 1) * D  # the state, in or out
        if mode == "step":
            return {"bytes": 2 * e * B * D + 2 * past + 4 * D * (n + 1), "flops": B * D * (2 * n + 4)}
        given = past if case["ragged"] else 0
        return {"bytes": 4 * e * B * L * D + past + given + 8 * D * (n + 1), "flops": B * L * D * (6 * n + 12)}
    if case["op"] == "scan":
        B, L, D, N, G = (case[k] for k in ("B", "L", "D", "N", "G"))
        tokens, shared, h = e * B * L * D, e * B * L * G * N, 4 * B * D * N
        params = 4 * D * (N + 2)
        given = h if mode == "step" or case["ragged"] else 0
        if mode != "train":
            return {"bytes": 4 * tokens + 2 * shared + params + h + given, "flops": 7 * B * L * D * N}
        return {"bytes": 8 * tokens + 4 * shared + 2 * params + h + given, "flops": 24 * B * L * D * N}
    if case["op"] == "norm":
        R, D = case["R"], case["D"]
        if mode == "serve":
            return {"bytes": 5 * e * R * D + 12 * D, "flops": 12 * R * D}
        return {"bytes": 10 * e * R * D + 24 * D, "flops": 40 * R * D}
    R, V, K = case["R"], case["V"], min(case["K"], case["V"])
    return {"bytes": 2 * e * R * V + (4 + e) * R * K + 16 * R, "flops": 10 * R * V}


# ----------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------
def _grads(of, gout, wrt):
    return torch.autograd.grad(of, wrt, gout)


def _exact_conv(s, case):
    n = s["w"].shape[1]
    x = (s["x"][:, None] if s["mode"] == "step" else s["x"]).double().requires_grad_()
    w, bias = s["w"].double().requires_grad_(), s["bias"].double().requires_grad_()
    B, L, D = x.shape
    past = s["state"].double() if s["state"] is not None else x.new_zeros(B, n - 1, D)
    count = [L] * B if s["lengths"] is None else s["lengths"].tolist()
    ys, states = [], []
    for b in range(B):
        seen = torch.cat([past[b], x[b, :count[b]]])
        p = bias.expand(count[b], D)
        for j in range(n):
            p = p + w[:, j] * seen[j:j + count[b]]
        ys.append(torch.cat([torch.nn.functional.silu(p), x.new_zeros(L - count[b], D)]))
        states.append(seen[count[b]:])
    y, state = torch.stack(ys), torch.stack(states)
    if s["mode"] == "step":
        return {"y": y[:, 0], "state": state}
    gx, gw, gbias = _grads(y, s["gy"].double(), (x, w, bias))
    return {"y": y, "state": state, "gx": gx, "gw": gw, "gbias": gbias}


def _exact_scan(s, case):
    step = s["mode"] == "step"
    train = s["mode"] == "train"
    B, L, D, N, G = (case[k] for k in ("B", "L", "D", "N", "G"))
    if L * B * D * N > 3e8 and train:  # every state of the sequence is kept for the gradient
        return None
    v = {k: (s[k][:, None] if step and k in ("x", "dt", "B", "C", "gate") else s[k]).double().requires_grad_(train)
         for k in ("x", "dt", "A", "B", "C", "skip", "gate", "dt_bias")}
    h = s["h0"].double() if s["h0"] is not None else torch.zeros((B, D, N), dtype=torch.float64, device=DEV)
    count = torch.full((B,), L, device=DEV) if s["lengths"] is None else s["lengths"]
    ys = []
    for t in range(L):
        live = (t < count)[:, None]
        delta = torch.nn.functional.softplus(v["dt"][:, t] + v["dt_bias"])
        Bt, Ct = (v[k][:, t, :, None].expand(B, G, D // G, N).reshape(B, D, N) for k in ("B", "C"))
        new = torch.exp(delta[..., None] * v["A"]) * h + (delta * v["x"][:, t])[..., None] * Bt
        h = torch.where(live[..., None], new, h)
        out = ((h * Ct).sum(-1) + v["skip"] * v["x"][:, t]) * torch.nn.functional.silu(v["gate"][:, t])
        ys.append(torch.where(live, out, 0.0))
    y = torch.stack(ys, 1)
    if step:
        return {"y": y[:, 0], "h": h}
    if not train:
        return {"y": y, "h": h}
    names = ("x", "dt", "A", "B", "C", "skip", "gate", "dt_bias")
    return {"y": y, "h": h, **{"g" + k: g for k, g in zip(names, _grads(y, s["gy"].double(), [v[k] for k in names]))}}


def _exact_norm(s, case):
    v = {k: s[k].double().requires_grad_() for k in ("x", "f", "gate", "scale", "w_post", "w_pre")}
    D = case["D"]
    act = torch.nn.functional.silu if s["act"] == "silu" else torch.sigmoid
    post = v["f"] / torch.sqrt(v["f"].square().sum(1, keepdim=True) / D + EPS) * v["w_post"]
    out = v["x"] + v["scale"] * act(v["gate"]) * post
    n = out / torch.sqrt(out.square().sum(1, keepdim=True) / D + EPS) * v["w_pre"]
    if s["mode"] == "serve":
        return {"out": out, "n": n}
    g = torch.autograd.grad([out, n], list(v.values()), [s["gout"].double(), s["gn"].double()])
    return {"out": out, "n": n, **{"g" + k: x for k, x in zip(v, g)}}


def _exact_distill(s, case):
    z, tau, alpha = s["z"].double().requires_grad_(), s["temperature"], s["alpha"]
    logp1, logpt = torch.log_softmax(z, 1), torch.log_softmax(z / tau, 1)
    has = s["idx"] >= 0
    rows = has.any(1)
    t = (s["teacher"].double() / tau).masked_fill(~has, -1e300)
    q = torch.where(rows[:, None], torch.softmax(t, 1), 0.0)
    logq = torch.where(q > 0, torch.log(q.clamp(min=1e-300)), 0.0)
    kl = (q * (logq - logpt.gather(1, s["idx"].long().clamp(min=0)))).sum(1)
    labelled = s["labels"] >= 0
    hard = torch.where(labelled, -logp1.gather(1, s["labels"].long().clamp(min=0)[:, None])[:, 0], 0.0)
    loss = s["weight"].double() * ((1 - alpha) * hard + alpha * tau ** 2 * kl)
    return {"loss": loss, "gz": _grads(loss, s["gloss"].double(), z)[0]}


EXACT = {"conv": _exact_conv, "scan": _exact_scan, "norm": _exact_norm, "distill": _exact_distill}


def exact(case, seed):
    got = EXACT[case["op"]](prepare(case, seed), case)
    return None if got is None else {k: v.detach() for k, v in got.items()}
