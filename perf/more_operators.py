"""What the rest of a transformer's training step is measured on: sizes, inputs and plain forms.

Beside rotary positions, attention, aggregation and orthogonalised updates a worker's gradient needs what
stands around attention: the norms before and after a block with the residual addition between them, the gated
feed-forward block, and the loss, here of a student that learns from a teacher's top logits.

  norm_fwd, norm_bwd       x' = x + scale act(gate) rms(f) post,  h = rms(x') pre, and the gradient of both
  ffn_fwd, ffn_bwd         y = (act(x Wg^T) * (x Wu^T)) Wd^T, and the gradients of x and the three weights
  distil_fwd, distil_bwd   per token mix tau^2 KL(p || softmax(z / tau)) + (1 - mix) (cross entropy of its label), and dz

`run` computes the plain form in fp32 (one rounding at the end) where `own` is false, and calls the
library where it is true.  `exact` states the same operators in fp64.
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the small example model's block end: an fp32 stream, one gain a channel as gate, short sequences: latency
        {"name": "norm fwd small f32", "op": "norm_fwd", "B": 16, "S": 96, "D": 128, "stream": "f32", "dtype": "bf16", "post": True, "gate": "channel", "by": "none", "pre": True, "scale": 1.0, "wide": 0},
        # a long batch of wide tokens, norms on both sides of the block, the block's own gate for every token
        {"name": "norm fwd wide bf16", "op": "norm_fwd", "B": 4, "S": 8192, "D": 4096, "stream": "bf16", "dtype": "bf16", "post": True, "gate": "token", "by": "sigmoid", "pre": True, "scale": 0.7, "wide": 0},
        # odd width and lengths, a gate for every sequence, the block's output a slice of something wider
        {"name": "norm bwd odd f16", "op": "norm_bwd", "B": 5, "S": 333, "D": 1001, "stream": "f16", "dtype": "f16", "post": True, "gate": "sequence", "by": "tanh", "pre": True, "scale": 0.5, "wide": 24},
        # the same wide batch's gradient with an fp32 stream
        {"name": "norm bwd wide f32", "op": "norm_bwd", "B": 4, "S": 8192, "D": 4096, "stream": "f32", "dtype": "bf16", "post": True, "gate": "channel", "by": "none", "pre": True, "scale": 0.7, "wide": 0},
        # sixteen single tokens through the encoder layer's block: the weights are what has to be read
        {"name": "ffn fwd tokens bf16", "op": "ffn_fwd", "T": 16, "D": 1024, "F": 4096, "act": "silu", "dtype": "bf16", "wide": 0},
        # a training batch of long contexts
        {"name": "ffn fwd long bf16", "op": "ffn_fwd", "T": 8192, "D": 4096, "F": 10944, "act": "silu", "dtype": "bf16", "wide": 0},
        # a few ragged sentences, odd token count, sides that end inside every tile
        {"name": "ffn bwd ragged f16", "op": "ffn_bwd", "T": 231, "D": 520, "F": 1368, "act": "gelu", "dtype": "f16", "wide": 40},
        # the encoder's own batch: 8 sentences of 512
        {"name": "ffn bwd encoder bf16", "op": "ffn_bwd", "T": 4096, "D": 1024, "F": 4096, "act": "gelu", "dtype": "bf16", "wide": 0},
        # the long contexts' gradient
        {"name": "ffn bwd long bf16", "op": "ffn_bwd", "T": 8192, "D": 4096, "F": 10944, "act": "silu", "dtype": "bf16", "wide": 0},
        # one sentence over an odd vocabulary, no labels: few rows, each of them long
        {"name": "distil fwd few f32", "op": "distil_fwd", "T": 19, "V": 50021, "K": 32, "tau": 2.0, "mix": 1.0, "labels": False, "dtype": "f32", "wide": 0},
        # a training batch over a large vocabulary, mixed with the labels' cross entropy
        {"name": "distil fwd batch bf16", "op": "distil_fwd", "T": 8192, "V": 131072, "K": 64, "tau": 2.0, "mix": 0.6, "labels": True, "dtype": "bf16", "wide": 0},
        # its gradient; the vocabulary ends inside the rows' padding
        {"name": "distil bwd batch bf16", "op": "distil_bwd", "T": 8192, "V": 131001, "K": 64, "tau": 2.0, "mix": 0.6, "labels": True, "dtype": "bf16", "wide": 71},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm_fwd", "norm_bwd", "norm_bwd", "ffn_fwd", "ffn_bwd", "ffn_bwd", "distil_fwd", "distil_bwd"))
    if op in ("norm_fwd", "norm_bwd"):
        D = _log(rng, 8, 8192)
        D = D // 8 * 8 if rng.random() < 0.6 else D
        B = _log(rng, 1, 64)
        S = max(1, min(_log(rng, 1, 8192), 2 ** 27 // (B * D)))
        dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
        post, pre = rng.random() < 0.75, rng.random() < 0.75
        gate = rng.choice(("none", "channel", "sequence", "token"))
        return {"op": op, "B": B, "S": S, "D": D, "stream": rng.choice((dtype, "f32")), "dtype": dtype, "post": post, "gate": gate,
                "by": "none" if gate == "none" else rng.choice(("none", "sigmoid", "tanh")), "pre": pre, "scale": rng.choice((1.0, 0.25)), "wide": rng.choice((0, 0, 8, 13))}
    if op in ("ffn_fwd", "ffn_bwd"):
        T, D, F = _log(rng, 1, 8192), 8 * _log(rng, 4, 512), 8 * _log(rng, 8, 1368)
        return {"op": op, "T": T, "D": D, "F": F, "act": rng.choice(("silu", "silu", "gelu", "gelu_tanh", "relu")), "dtype": rng.choice(("bf16", "bf16", "f16")),
                "wide": rng.choice((0, 0, 8, 64))}
    V = _log(rng, 100, 131072)
    T = max(1, min(_log(rng, 1, 8192), 2 ** 29 // V))
    labels = rng.random() < 0.5
    return {"op": op, "T": T, "V": V, "K": min(V, _log(rng, 1, 128)), "tau": rng.choice((1.0, 2.0, 0.5, 3.7)), "mix": 0.7 if labels else 1.0, "labels": labels,
            "dtype": rng.choice(("bf16", "f16", "f32")), "wide": rng.choice((0, 0, 3, 64))}


# ---------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------
def _rand(g, shape, dtype, wide=0, scale=1.0):
    """Normal values; `wide` more columns lie behind those of every row."""
    full = (scale * torch.randn((*shape[:-1], shape[-1] + wide), generator=g, device="cuda")).to(dtype)
    return full[..., :shape[-1]] if wide else full


def _prepare_norm(case, g):
    B, S, D, t = case["B"], case["S"], case["D"], TYPES[case["dtype"]]
    st = {"x": _rand(g, (B, S, D), TYPES[case["stream"]], scale=2.0), "f": _rand(g, (B, S, D), t, case["wide"], 0.5)}
    # gains lie around one, gates around a small value
    st["post"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")) if case["post"] else None
    st["pre"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")) if case["pre"] else None
    shape = {"none": None, "channel": (D,), "sequence": (B, D), "token": (B, S, D)}[case["gate"]]
    st["gate"] = None if shape is None else 0.3 + _rand(g, shape, t if case["gate"] == "token" else torch.float32)
    if case["op"] == "norm_bwd":
        out, _, rows = _norm(case, st["x"], st["f"], st["post"], st["gate"], st["pre"])      # the forward pass has been
        st["out"], st["rows"] = out, rows
        st["dout"] = _rand(g, (B, S, D), TYPES[case["stream"]], scale=0.1)
        st["dnormed"] = _rand(g, (B, S, D), t, scale=0.1) if case["pre"] else None
    return st


def _prepare_ffn(case, g):
    T, D, F, t = case["T"], case["D"], case["F"], TYPES[case["dtype"]]
    st = {"x": _rand(g, (T, D), t, case["wide"])}
    st["wg"], st["wu"] = (_rand(g, (F, D), t, scale=D ** -0.5) for _ in range(2))
    st["wd"] = _rand(g, (D, F), t, scale=F ** -0.5)
    if case["op"] == "ffn_bwd":
        x = st["x"].float()
        st["g"], st["u"] = (x @ st["wg"].float().T).to(t), (x @ st["wu"].float().T).to(t)     # the forward pass has been
        st["dy"] = _rand(g, (T, D), t, scale=0.1)
    return st


def _prepare_distil(case, g):
    T, V, K = case["T"], case["V"], case["K"]
    st = {"z": _rand(g, (T, V), TYPES[case["dtype"]], case["wide"], 3.0)}
    ids, top = [], []
    for at in range(0, T, 512):                         # a teacher that agrees with the student in part
        full = 0.7 * st["z"][at:at + 512].float() + 2.5 * torch.randn((min(512, T - at), V), generator=g, device="cuda")
        v, i = full.topk(K)
        top.append(v)
        ids.append(i)
    st["ids"], st["top"] = torch.cat(ids), torch.cat(top)
    # padding tokens have no entry at all, and some tokens' lists are short
    kept = torch.randint(1, K + 1, (T, 1), generator=g, device="cuda")
    kept = torch.where(torch.rand((T, 1), generator=g, device="cuda") < 0.5, kept, K)
    padding = torch.rand((T, 1), generator=g, device="cuda") < (0.1 if T > 1 else 0.0)
    hidden = (torch.arange(K, device="cuda") >= kept) | padding
    st["ids"] = st["ids"].masked_fill(hidden, -1)
    st["labels"] = None
    if case["labels"]:
        st["labels"] = torch.randint(0, V, (T,), generator=g, device="cuda").masked_fill(padding[:, 0], -100)
    if case["op"] == "distil_bwd":
        st["rows"] = _distil(case, st["z"], st["ids"], st["top"], st["labels"])[1]      # the forward pass has been
        st["dloss"] = torch.rand(T, generator=g, device="cuda") + 0.5
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = {"norm": _prepare_norm, "ffn": _prepare_ffn, "distil": _prepare_distil}[case["op"].split("_")[0]](case, g)
    st["case"] = dict(case)
    return st


# ---------------------------------------------------------------------------------------------------------
# plain forms, fp32
# ---------------------------------------------------------------------------------------------------------
def _gate(case, gate):
    """(act(gate), its derivative), broadcast over the tokens."""
    if gate is None:
        return 1.0, 0.0
    a = gate.float()
    a = a[:, None] if case["gate"] == "sequence" else a
    if case["by"] == "sigmoid":
        s = 1 / (1 + (-a).exp())
        return s, s * (1 - s)
    if case["by"] == "tanh":
        s = torch.tanh(a)
        return s, 1 - s * s
    return a, torch.ones_like(a)


def _norm(case, x, f, post, gate, pre):
    n, rf, rx, h = f.float(), None, None, None
    if post is not None:
        rf = (n.square().mean(-1, keepdim=True) + EPS).rsqrt()
        n = n * rf * post
    new = x.float() + case["scale"] * _gate(case, gate)[0] * n
    if pre is not None:
        rx = (new.square().mean(-1, keepdim=True) + EPS).rsqrt()
        h = (new * rx * pre).to(f.dtype)
    zeros = torch.zeros(x.shape[:2], device=x.device)
    rows = torch.stack([zeros if r is None else r.squeeze(-1) for r in (rf, rx)])
    return new.to(x.dtype), h, rows


def _norm_backward(case, st):
    f, post, gate, pre, t = st["f"].float(), st["post"], st["gate"], st["pre"], st["dout"].float()
    rf, rx = st["rows"][0][..., None], st["rows"][1][..., None]
    dpre = dpost = dgate = None
    if pre is not None:
        dh, xh = st["dnormed"].float(), st["out"].float() * rx
        a = dh * pre
        t = t + rx * (a - xh * (a * xh).mean(-1, keepdim=True))
        dpre = (dh * xh).sum((0, 1))
    n = f * rf if post is not None else f
    c, slope = _gate(case, gate)
    c = case["scale"] * c
    e = c * t
    if post is not None:
        dpost = (e * n).sum((0, 1))
        e = e * post
        df = rf * (e - n * (e * n).mean(-1, keepdim=True))
    else:
        df = e
    if gate is not None:
        d = case["scale"] * slope * t * n * (1.0 if post is None else post)
        dgate = {"channel": lambda: d.sum((0, 1)), "sequence": lambda: d.sum(1), "token": lambda: d}[case["gate"]]().to(gate.dtype)
    return t.to(st["out"].dtype), df.to(st["f"].dtype), dgate, dpost, dpre


def _act(case, g):
    """(act(g), act'(g))"""
    if case["act"] == "silu":
        s = 1 / (1 + (-g).exp())
        return g * s, s * (1 + g * (1 - s))
    if case["act"] == "gelu":
        phi = 0.5 * (1 + torch.erf(g * 2 ** -0.5))
        return g * phi, phi + g * (-0.5 * g * g).exp() / math.sqrt(2 * math.pi)
    if case["act"] == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        th = torch.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + th), 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * k * (1 + 3 * 0.044715 * g * g)
    return g.clamp_min(0), (g > 0).float()


def _ffn(case, st):
    x = st["x"].float()
    g, u = x @ st["wg"].float().T, x @ st["wu"].float().T
    y = (_act(case, g)[0] * u) @ st["wd"].float().T
    t = st["x"].dtype
    return y.to(t), g.to(t), u.to(t)


def _ffn_backward(case, st):
    x, g, u, dy = (st[k].float() for k in ("x", "g", "u", "dy"))
    a, slope = _act(case, g)
    dh = dy @ st["wd"].float()
    dg, du = dh * u * slope, dh * a
    dx = dg @ st["wg"].float() + du @ st["wu"].float()
    return tuple(v.to(st["x"].dtype) for v in (dx, dg.T @ x, du.T @ x, dy.T @ (a * u)))


def _teacher(case, ids, top):
    """(probabilities of a row's kept entries, zeros elsewhere; whether the row has any)"""
    t = (top.float() / case["tau"]).masked_fill(ids < 0, -math.inf)
    has = (ids >= 0).any(1, keepdim=True)
    e = (t - t.amax(1, keepdim=True).clamp_min(-3e38)).exp()
    return e / e.sum(1, keepdim=True).clamp_min(1e-30), has


def _lse(z):
    m = z.amax(1, keepdim=True)
    return m + (z - m).exp().sum(1, keepdim=True).log()


def _distil(case, z, ids, top, labels):
    z, tau = z.float(), case["tau"]
    p, has = _teacher(case, ids, top)
    L = _lse(z / tau)
    logq = z.gather(1, ids.clamp_min(0)) / tau - L
    loss = case["mix"] * tau ** 2 * (p * (p.clamp_min(1e-38).log() - logq)).sum(1, keepdim=True) * has
    rows = [L * has, torch.zeros_like(L)]
    if labels is not None:
        some = (labels >= 0)[:, None]
        L1 = _lse(z)
        loss = loss + (1 - case["mix"]) * some * (L1 - z.gather(1, labels.clamp_min(0)[:, None]))
        rows = [L * (has | some), L1 * (has | some)]
    return loss.squeeze(1), torch.cat(rows, 1).T.contiguous()


def _distil_backward(case, st):
    z, ids, labels, tau = st["z"].float(), st["ids"], st["labels"], case["tau"]
    p, has = _teacher(case, ids, st["top"])
    d = (z / tau - st["rows"][0][:, None]).exp() * has
    d.scatter_add_(1, ids.clamp_min(0), -p)
    d *= case["mix"] * tau
    if labels is not None:
        some = (labels >= 0)[:, None]
        d += (1 - case["mix"]) * some * (z - st["rows"][1][:, None]).exp()
        d.scatter_add_(1, labels.clamp_min(0)[:, None], -(1 - case["mix"]) * some.float())
    return (st["dloss"][:, None] * d).to(st["z"].dtype)


def run(state):
    case, st = state["case"], state
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd"):
        how = {"post": st["post"], "gate": st["gate"], "gate_by": None if case["by"] == "none" else case["by"], "scale": case["scale"], "pre": st["pre"]}
        if op == "norm_fwd":
            if own:
                from paper_2411_03742_b200 import residual_norm_forward
                made = residual_norm_forward(st["x"], st["f"], eps=EPS, **how)
            else:
                made = _norm(case, st["x"], st["f"], st["post"], st["gate"], st["pre"])
        elif own:
            from paper_2411_03742_b200 import residual_norm_backward
            made = residual_norm_backward(st["dout"], st["dnormed"], st["out"], st["f"], st["rows"], **how)
        else:
            made = _norm_backward(case, st)
        return tuple(t for t in made if t is not None)
    if op == "ffn_fwd":
        if own:
            from paper_2411_03742_b200 import feedforward_forward
            return feedforward_forward(st["x"], st["wg"], st["wu"], st["wd"], act=case["act"])
        return _ffn(case, st)
    if op == "ffn_bwd":
        if own:
            from paper_2411_03742_b200 import feedforward_backward
            return feedforward_backward(st["dy"], st["x"], st["wg"], st["wu"], st["wd"], st["g"], st["u"], act=case["act"])
        return _ffn_backward(case, st)
    how = {"temperature": case["tau"], "labels": st["labels"], "mix": case["mix"]}
    if op == "distil_fwd":
        if own:
            from paper_2411_03742_b200 import distill_forward
            return distill_forward(st["z"], st["ids"], st["top"], **how)
        return _distil(case, st["z"], st["ids"], st["top"], st["labels"])
    if own:
        from paper_2411_03742_b200 import distill_backward
        return distill_backward(st["dloss"], st["z"], st["ids"], st["top"], st["rows"], **how)
    return _distil_backward(case, st)


# ---------------------------------------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("norm_fwd", "norm_bwd"):
        n, s, b = case["B"] * case["S"] * case["D"], SIZE[case["stream"]], SIZE[case["dtype"]]
        token = b * n if case["gate"] == "token" else 0
        small = 4 * case["D"] * (case["post"] + case["pre"] + {"none": 0, "token": 0, "channel": 1, "sequence": case["B"]}[case["gate"]])
        rows = 4 * case["B"] * case["S"] * (case["post"] + case["pre"])
        h = b * n if case["pre"] else 0
        if op == "norm_fwd":
            return {"bytes": n * (2 * s + b) + h + token + small + rows, "flops": 10 * n}
        # dout, out (for its norm), dx; f, df; the gate and its gradient
        return {"bytes": n * (2 * s + 2 * b) + (h + s * n if case["pre"] else 0) + 2 * token + 2 * small + rows, "flops": 25 * n}
    if op in ("ffn_fwd", "ffn_bwd"):
        T, D, F = case["T"], case["D"], case["F"]
        if op == "ffn_fwd":
            return {"bytes": 2 * (2 * T * D + 2 * T * F + 3 * D * F), "flops": 6 * T * D * F}
        return {"bytes": 2 * (3 * T * D + 2 * T * F + 6 * D * F), "flops": 12 * T * D * F}
    T, V, K = case["T"], case["V"], case["K"]
    b = SIZE[case["dtype"]]
    top = T * K * 12 + T * 12 + (8 * T if case["labels"] else 0)
    exps = 2 if case["labels"] and case["tau"] != 1.0 else 1
    return {"bytes": (1 if op == "distil_fwd" else 2) * b * T * V + top, "flops": T * V * (2 + 2 * exps)}


def _exact_norm(case, st):
    f, x = st["f"].double(), st["x"].double()
    post = torch.ones((), dtype=torch.float64, device="cuda") if st["post"] is None else st["post"].double()
    gate = None if st["gate"] is None else st["gate"].double()
    if gate is not None and case["gate"] == "sequence":
        gate = gate.unsqueeze(1).expand(-1, case["S"], -1)
    opened = {"none": lambda v: v, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[case["by"]]
    factor = case["scale"] if gate is None else case["scale"] * opened(gate)
    back = case["op"] == "norm_bwd"
    if back:
        rf = st["rows"][0].double().unsqueeze(-1)
    else:
        rf = 1.0 / torch.sqrt((f * f).sum(-1, keepdim=True) / case["D"] + EPS)
    unit = f if st["post"] is None else f * rf
    if not back:
        new = x + factor * unit * post
        if st["pre"] is None:
            normed, rx = None, torch.zeros_like(rf)
        else:
            rx = 1.0 / torch.sqrt((new * new).sum(-1, keepdim=True) / case["D"] + EPS)
            normed = new * rx * st["pre"].double()
        rows = torch.cat([torch.zeros_like(rf) if st["post"] is None else rf, rx], -1).permute(2, 0, 1)
        return tuple(v for v in (new, normed, rows) if v is not None)
    total, dpre = st["dout"].double(), None
    if st["pre"] is not None:
        rx = st["rows"][1].double().unsqueeze(-1)
        hat, dh = st["out"].double() * rx, st["dnormed"].double()
        inner = torch.einsum("bsd,bsd,d->bs", dh, hat, st["pre"].double()) / case["D"]
        total = total + rx * dh * st["pre"].double() - rx * hat * inner.unsqueeze(-1)
        dpre = torch.einsum("bsd,bsd->d", dh, hat)
    by_unit = total * factor * post
    if st["post"] is None:
        df = by_unit
    else:
        df = rf * by_unit - rf * unit * torch.einsum("bsd,bsd->bs", by_unit, unit).unsqueeze(-1) / case["D"]
    dgate = None
    if gate is not None:
        slope = {"none": lambda v: torch.ones_like(v), "sigmoid": lambda v: torch.sigmoid(v) * torch.sigmoid(-v), "tanh": lambda v: torch.cosh(v) ** -2}[case["by"]](gate)
        d = case["scale"] * total * unit * post * slope
        dgate = {"channel": "bsd->d", "sequence": "bsd->bd", "token": "bsd->bsd"}[case["gate"]]
        dgate = torch.einsum(dgate, d)
    dpost = None if st["post"] is None else torch.einsum("bsd,bsd->d", total * factor, unit)
    return tuple(v for v in (total, df, dgate, dpost, dpre) if v is not None)


def _exact_ffn(case, st):
    import torch.nn.functional as fn
    act = {"silu": fn.silu, "gelu": fn.gelu, "gelu_tanh": lambda v: fn.gelu(v, approximate="tanh"), "relu": fn.relu}[case["act"]]
    x, wg, wu, wd = (st[k].double() for k in ("x", "wg", "wu", "wd"))
    if case["op"] == "ffn_fwd":
        g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
        return torch.mm(act(g).mul_(u), wd.t()), g, u
    dy = st["dy"].double()
    g, u = st["g"].double().requires_grad_(), st["u"].double().requires_grad_()
    h = act(g) * u
    dg, du = torch.autograd.grad(h, (g, u), torch.mm(dy, wd))
    return torch.addmm(torch.mm(dg, wg), du, wu), torch.mm(dg.t(), x), torch.mm(du.t(), x), torch.mm(dy.t(), h.detach())


def _exact_distil(case, st):
    T, V, K, tau, mix = case["T"], case["V"], case["K"], case["tau"], case["mix"]
    back = case["op"] == "distil_bwd"
    losses, rows, dz = [], [], []
    for at in range(0, T, 256):                         # a few tokens at a time
        part = slice(at, min(at + 256, T))
        z, ids, top = st["z"][part].double(), st["ids"][part], st["top"][part].double()
        label = st["labels"][part] if case["labels"] else torch.full((z.shape[0],), -1, device="cuda")
        kept, known = ids.ge(0), label.ge(0)
        taught = kept.any(1)
        log_p = torch.where(kept, top / tau, torch.full_like(top, -math.inf))
        log_p = log_p - torch.where(taught, torch.logsumexp(log_p, 1), torch.zeros_like(log_p[:, 0]))[:, None]
        p = torch.exp(log_p)
        n = torch.arange(z.shape[0], device="cuda")
        if not back:
            wide, plain = torch.logsumexp(z / tau, 1), torch.logsumexp(z, 1)
            there = torch.where(kept, torch.take_along_dim(z, ids.clamp(min=0), 1) / tau - wide[:, None], torch.zeros_like(p))
            kl = torch.where(kept, p * (torch.where(kept, log_p, torch.zeros_like(p)) - there), torch.zeros_like(p)).sum(1)
            hard = torch.where(known, plain - z[n, label.clamp(min=0)], torch.zeros_like(plain))
            losses.append(mix * tau * tau * torch.where(taught, kl, torch.zeros_like(kl)) + (1.0 - mix) * hard)
            used = (taught | known).double()
            rows.append(torch.stack([wide * used, plain * used * float(case["labels"])]))
            continue
        d = torch.exp(z / tau - st["rows"][0][part].double()[:, None]) * (mix * tau * taught.double())[:, None]
        target = torch.zeros_like(d)
        target.scatter_add_(1, ids.clamp(min=0), mix * tau * torch.where(kept, p, torch.zeros_like(p)))
        if case["labels"]:
            d += torch.exp(z - st["rows"][1][part].double()[:, None]) * ((1.0 - mix) * known.double())[:, None]
            target[n, label.clamp(min=0)] += (1.0 - mix) * known.double()
        dz.append((d - target) * st["dloss"][part].double()[:, None])
    return torch.cat(dz) if back else (torch.cat(losses), torch.cat(rows, 1))


def exact(case, seed):
    st = prepare(case, seed)
    return {"norm": _exact_norm, "ffn": _exact_ffn, "distil": _exact_distil}[case["op"].split("_")[0]](case, st)
