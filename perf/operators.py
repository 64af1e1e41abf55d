"""What the training operators beside the aggregation are measured on: sizes, inputs and plain forms.

The aggregation turns N worker gradients into one direction.  The operators here stand on both sides
of it in a training step of a transformer: rotary positions and attention with its gradient, which
produce a worker's gradient, and the orthogonalisation of the aggregated direction, matrix by matrix,
which turns it into an update.

  orth       out = NS(update): Newton-Schulz polynomial products on every weight matrix of a flat vector
  attn_fwd   O = softmax(scale Q K^T + mask) V and the rows' log-sum-exp
  attn_bwd   dQ, dK, dV from dO, with the probabilities recomputed from the log-sum-exp
  rope       rotary positions, forward and gradient, half and interleaved pairs, scaled frequencies

`run` computes the plain form in fp32 (one rounding at the end) where `own` is false, and calls the
library where it is true.  `exact` states the same operators in fp64.
"""
import math

import torch

own = False

STEPS = 5
COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# The matrices of one encoder layer of the BERT-Large-sized workload: four attention projections, two feed-forward ones.
LAYER = "1024x1024,1024x1024,1024x1024,1024x1024,4096x1024,1024x4096"


def listed():
    return [
        # one small projection matrix: nothing but latency
        {"name": "orth one 96x200 f32", "op": "orth", "shapes": "96x200", "dtype": "f32", "gap": 0},
        # one encoder layer of the BERT-Large-sized workload, as a job that overlaps layers calls it
        {"name": "orth layer bf16", "op": "orth", "shapes": LAYER, "dtype": "bf16", "gap": 1024},
        # a ragged flat vector: odd sides, tall and wide, matrices at odd offsets between biases
        {"name": "orth ragged f32", "op": "orth", "shapes": "1001x333,77x1500,640x641,31x31,513x2049,1200x1200,129x257,1999x65", "dtype": "f32", "gap": 37},
        # twelve layers at once: half the BERT-Large-sized vector in one call
        {"name": "orth 12 layers bf16", "op": "orth", "shapes": ",".join([LAYER] * 12), "dtype": "bf16", "gap": 1024},
        # the encoder's own attention at its pre-training length, padded sentences
        {"name": "attn fwd encoder", "op": "attn_fwd", "B": 8, "Hq": 16, "Hkv": 16, "Sq": 512, "Sk": 512, "D": 64, "causal": False, "lens": True, "packed": True},
        # a long causal context with shared key heads
        {"name": "attn fwd long causal", "op": "attn_fwd", "B": 1, "Hq": 32, "Hkv": 8, "Sq": 8192, "Sk": 8192, "D": 128, "causal": True, "lens": False, "packed": False},
        # a handful of short sentences: latency, odd lengths, one sentence with no key at all
        {"name": "attn bwd short odd", "op": "attn_bwd", "B": 3, "Hq": 4, "Hkv": 2, "Sq": 77, "Sk": 91, "D": 40, "causal": False, "lens": True, "packed": False},
        # the encoder's gradient
        {"name": "attn bwd encoder", "op": "attn_bwd", "B": 8, "Hq": 16, "Hkv": 16, "Sq": 512, "Sk": 512, "D": 64, "causal": False, "lens": True, "packed": True},
        # the long causal context's gradient, four query heads to a key head
        {"name": "attn bwd long causal", "op": "attn_bwd", "B": 1, "Hq": 32, "Hkv": 8, "Sq": 8192, "Sk": 8192, "D": 128, "causal": True, "lens": False, "packed": False},
        # single new tokens of sixteen sequences at long positions
        {"name": "rope tokens bf16", "op": "rope", "B": 16, "S": 1, "H": 40, "D": 128, "rot": 128, "interleaved": False, "scaling": "none", "dtype": "bf16", "inverse": False, "far": 30000},
        # an odd length, a part of an odd head rotated, adjacent pairs, fp32
        {"name": "rope part interleaved f32", "op": "rope", "B": 3, "S": 1001, "H": 12, "D": 80, "rot": 32, "interleaved": True, "scaling": "linear", "dtype": "f32", "inverse": False, "far": 0},
        # the gradient over a context extended sixteen-fold
        {"name": "rope long gradient bf16", "op": "rope", "B": 1, "S": 65536, "H": 40, "D": 128, "rot": 128, "interleaved": False, "scaling": "yarn", "dtype": "bf16", "inverse": True, "far": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("orth", "orth", "attn_fwd", "attn_bwd", "attn_bwd", "rope"))
    if op == "orth":
        shapes, left = [], 1.0e11                       # multiply-adds of one polynomial step, well under the largest listed case
        for _ in range(_log(rng, 1, 24)):
            m, n = _log(rng, 24, 4096), _log(rng, 24, 4096)
            cost = float(min(m, n)) ** 2 * max(m, n)
            if cost <= left:
                shapes.append("%dx%d" % (m, n))
                left -= cost
        return {"op": op, "shapes": ",".join(shapes or ["64x64"]), "dtype": rng.choice(("f32", "bf16")), "gap": rng.choice((0, 5, 1024))}
    if op == "rope":
        D = 8 * rng.randint(4, 16)
        return {"op": op, "B": _log(rng, 1, 16), "S": _log(rng, 1, 4096), "H": rng.randint(1, 40), "D": D, "rot": rng.choice((D, 8 * rng.randint(2, D // 8))),
                "interleaved": rng.random() < 0.5, "scaling": rng.choice(("none", "linear", "ntk", "yarn")), "dtype": rng.choice(("f32", "bf16")),
                "inverse": rng.random() < 0.5, "far": rng.choice((0, 30000))}
    Hkv = rng.choice((1, 2, 4, 8))
    Hq = Hkv * rng.choice((1, 2, 4))
    # one key's softmax has no gradient, only rounding noise: gradients are drawn from 16 tokens on
    D, Sq = 8 * rng.randint(4, 16), _log(rng, 1 if op == "attn_fwd" else 16, 4000)
    causal, packed = rng.random() < 0.5, rng.random() < 0.5
    Sk = Sq if packed or rng.random() < 0.5 else _log(rng, 16, 4000)
    B = max(1, min(_log(rng, 1, 16), 2 ** 29 // (Hq * Sq * Sk)))
    return {"op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "Sk": Sk, "D": D, "causal": causal, "lens": rng.random() < 0.5, "packed": packed}


# ---------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------
def _layout(case):
    """[(rows, cols, offset)] of the matrices in the flat vector and its length: `gap` elements (a bias, a norm's weights) behind each."""
    at, places = 0, []
    for s in case["shapes"].split(","):
        m, n = (int(x) for x in s.split("x"))
        places.append((m, n, at))
        at += m * n + case["gap"]
    return places, at


def _lens(case, seed):
    """Key lengths of a padded batch: from none to all."""
    g = torch.Generator().manual_seed(seed + 7)
    lens = torch.randint(0, case["Sk"] + 1, (case["B"],), generator=g)
    lens[0] = case["Sk"]
    if case["B"] > 1:
        lens[1] = 0
    return lens.to(torch.int32)


def _qkv(case, seed, dev):
    g = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    if case["packed"]:                                  # one projection's output: q, k and v are slices of its heads
        qkv = torch.randn((B, case["Sq"], Hq + 2 * Hkv, D), generator=g, device=dev).to(torch.bfloat16)
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    else:
        q = torch.randn((B, case["Sq"], Hq, D), generator=g, device=dev).to(torch.bfloat16)
        k = torch.randn((B, case["Sk"], Hkv, D), generator=g, device=dev).to(torch.bfloat16)
        v = torch.randn((B, case["Sk"], Hkv, D), generator=g, device=dev).to(torch.bfloat16)
    lens = _lens(case, seed).to(dev) if case["lens"] else None
    dout = torch.randn((B, case["Sq"], Hq, D), generator=g, device=dev).to(torch.bfloat16)
    return q, k, v, lens, dout


def _frequencies(case):
    """Angles per position of the rotated pairs and the factor on the rotated values, in fp64."""
    r, base, scaling = case["rot"], 10000.0, case["scaling"]
    if scaling == "ntk":                                # a larger base: the slowest pair turns `factor` times slower, the fastest as before
        base = base * 8.0 ** (r / (r - 2.0))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "yarn":                               # by parts: pairs that turn often keep their angle, slow ones are interpolated
        factor, length = 16.0, 4096.0
        lo = max(math.floor(r * math.log(length / (32.0 * 2 * math.pi)) / (2 * math.log(base))), 0)
        hi = min(math.ceil(r * math.log(length / (1.0 * 2 * math.pi)) / (2 * math.log(base))), r - 1)
        ramp = ((torch.arange(r // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    return f, 1.0


SCALING = {"none": None, "linear": ("linear", 4.0), "ntk": ("ntk", 8.0), "yarn": ("yarn", 16.0, 4096)}


def _positions(case, seed, dev):
    """Two documents in a row of the batch: positions start anew in the middle; `far` tokens lie before the first."""
    g = torch.Generator().manual_seed(seed + 3)
    p = torch.arange(case["S"]).repeat(case["B"], 1)
    cut = torch.randint(0, case["S"] + 1, (case["B"], 1), generator=g)
    p = torch.where(p >= cut, p - cut, p)
    if case["far"]:
        p = p + torch.randint(0, case["far"], (case["B"], 1), generator=g)
    return p.to(torch.int32).to(dev)


def prepare(case, seed):
    dev = torch.device("cuda")
    st = {"case": dict(case)}
    if case["op"] == "orth":
        places, d = _layout(case)
        g = torch.Generator(device=dev).manual_seed(seed)
        u = 1e-3 * torch.randn(d, generator=g, device=dev)              # a step's noise ...
        for m, n, at in places:                                         # ... on a few directions that the workers agree on
            a, b = torch.randn((m, 8), generator=g, device=dev), torch.randn((8, n), generator=g, device=dev)
            u[at:at + m * n] += 5e-4 * (a @ b).reshape(-1)
        st["update"], st["places"] = u.to(TYPES[case["dtype"]]), places
        st["out"] = torch.zeros_like(st["update"])                      # what lies between the matrices stays as it is
        if own:
            from paper_2411_03742_b200 import Orthogonalizer
            st["plan"] = Orthogonalizer([(m, n) for m, n, _ in places], case["dtype"], offsets=[at for _, _, at in places], d=d, steps=STEPS, coeffs=COEFFS, eps=EPS)
    elif case["op"] == "rope":
        g = torch.Generator(device=dev).manual_seed(seed)
        st["x"] = torch.randn((case["B"], case["S"], case["H"], case["D"]), generator=g, device=dev).to(TYPES[case["dtype"]])
        st["positions"] = _positions(case, seed, dev)
        if own:
            from paper_2411_03742_b200 import Rope
            st["plan"] = Rope(case["rot"], base=10000.0, interleaved=case["interleaved"], scaling=SCALING[case["scaling"]])
        else:                                                           # the cosines and sines of all positions, kept between calls
            f, factor = _frequencies(case)
            angle = torch.arange(case["S"] + case["far"], dtype=torch.float64, device=dev)[:, None] * f.to(dev)
            st["cos"], st["sin"] = (factor * angle.cos()).float(), (factor * angle.sin()).float()
    else:
        st["q"], st["k"], st["v"], st["lens"], st["dout"] = _qkv(case, seed, dev)
        if case["op"] == "attn_bwd":                                    # the forward pass has been
            st["out"], st["lse"] = _attention(case, st["q"], st["k"], st["v"], st["lens"])
    return st


# ---------------------------------------------------------------------------------------------------------
# plain forms, fp32
# ---------------------------------------------------------------------------------------------------------
def _orthogonalise(case, update, places, out):
    a, b, c = COEFFS
    shapes = {}
    for m, n, at in places:
        shapes.setdefault((m, n), []).append(at)
    for (m, n), ats in shapes.items():                                  # equal matrices together
        x = torch.stack([update[at:at + m * n].view(m, n) for at in ats]).float()
        x = x.mT if m > n else x
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(STEPS):
            s = x @ x.mT
            x = a * x + (b * s + c * (s @ s)) @ x
        x = (x.mT if m > n else x).to(out.dtype)
        for i, at in enumerate(ats):
            out[at:at + m * n] = x[i].reshape(-1)
    return out


def _masked_scores(case, q, k, lens):
    """scale Q K^T with -inf where a query does not see a key; shapes B, H, S, D."""
    s = (q @ k.mT) / math.sqrt(case["D"])
    j = torch.arange(case["Sk"], device=s.device)
    if lens is not None:
        s.masked_fill_((j >= lens[:, None])[:, None, None], -math.inf)
    if case["causal"]:                                                  # the last query sees the last key
        i = torch.arange(case["Sq"], device=s.device)[:, None]
        s.masked_fill_(j > i + (case["Sk"] - case["Sq"]), -math.inf)
    return s


def _heads(x, groups=1):
    x = x.float().transpose(1, 2)
    return x.repeat_interleave(groups, 1) if groups > 1 else x


def _attention(case, q, k, v, lens):
    r = case["Hq"] // case["Hkv"]
    s = _masked_scores(case, _heads(q), _heads(k, r), lens)
    top = s.amax(-1, keepdim=True).clamp_min(-3e38)                     # a row that sees no key: its exponentials are all zero
    p = (s - top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ _heads(v, r)) / total.clamp_min(1e-30)
    lse = torch.where(total > 0, top + total.log(), -math.inf).squeeze(-1)
    return out.transpose(1, 2).to(q.dtype).contiguous(), lse


def _attention_backward(case, q, k, v, lens, out, lse, dout):
    B, r, scale = case["B"], case["Hq"] // case["Hkv"], 1.0 / math.sqrt(case["D"])
    qf, kf, vf, do = _heads(q), _heads(k, r), _heads(v, r), _heads(dout)
    p = (_masked_scores(case, qf, kf, lens) - lse.clamp_min(-3e38)[..., None]).exp_()
    dv = p.mT @ do
    ds = p.mul_((do @ vf.mT) - (do * _heads(out)).sum(-1, keepdim=True))
    dq, dk = scale * (ds @ kf), scale * (ds.mT @ qf)
    dk, dv = (x.view(B, case["Hkv"], r, case["Sk"], case["D"]).sum(2) for x in (dk, dv))
    return tuple(x.transpose(1, 2).to(q.dtype).contiguous() for x in (dq, dk, dv))


def _rotate(case, x, positions, cos, sin):
    r = case["rot"]
    cos, sin = (t[positions.long()][:, :, None] for t in (cos, sin))
    sin = -sin if case["inverse"] else sin
    f = x.float()
    if case["interleaved"]:
        a, b = f[..., 0:r:2], f[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = f[..., :r // 2], f[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, f[..., r:]), -1).to(x.dtype)


def run(state):
    case = state["case"]
    if case["op"] == "orth":
        if own:
            state["plan"].apply(state["update"], state["out"])
            return state["out"]
        return _orthogonalise(case, state["update"], state["places"], state["out"])
    if case["op"] == "rope":
        if own:
            return state["plan"].apply(state["x"], state["positions"], inverse=case["inverse"])
        return _rotate(case, state["x"], state["positions"], state["cos"], state["sin"])
    if case["op"] == "attn_fwd":
        if own:
            from paper_2411_03742_b200 import attention_forward
            return attention_forward(state["q"], state["k"], state["v"], causal=case["causal"], kv_lens=state["lens"])
        return _attention(case, state["q"], state["k"], state["v"], state["lens"])
    if own:
        from paper_2411_03742_b200 import attention_backward
        return attention_backward(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], causal=case["causal"], kv_lens=state["lens"])
    return _attention_backward(case, state["q"], state["k"], state["v"], state["lens"], state["out"], state["lse"], state["dout"])


# ---------------------------------------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------
def _pairs(case):
    """Query-key pairs that the mask leaves, over all batches, of one head (padded lengths: the mean of the draw, half)."""
    Sq, Sk = case["Sq"], case["Sk"]
    if case["causal"]:
        seen = sum(min(max(i + 1 + Sk - Sq, 0), Sk) for i in range(Sq))
    else:
        seen = Sq * Sk
    return case["B"] * seen * (0.5 if case["lens"] else 1.0)


def work(case):
    if case["op"] == "orth":
        size = 4 if case["dtype"] == "f32" else 2
        flops = elements = 0
        for m, n, _ in _layout(case)[0]:
            r, l = min(m, n), max(m, n)
            # per step: X X^T and its square, symmetric (half the products each), then a full product with X
            flops += STEPS * (r * r * l + r * r * r + 2 * r * r * l)
            elements += m * n
        return {"bytes": 2 * size * elements, "flops": flops}
    if case["op"] == "rope":
        n = case["B"] * case["S"]
        return {"bytes": 2 * n * case["H"] * case["D"] * (4 if case["dtype"] == "f32" else 2) + 4 * n, "flops": 3 * n * case["H"] * case["rot"]}
    B, D = case["B"], case["D"]
    q, kv, rows = B * case["Sq"] * case["Hq"] * D, B * case["Sk"] * case["Hkv"] * D, B * case["Sq"] * case["Hq"]
    if case["op"] == "attn_fwd":
        return {"bytes": 2 * (2 * q + 2 * kv) + 4 * rows, "flops": 4 * D * case["Hq"] * _pairs(case)}
    return {"bytes": 2 * (4 * q + 4 * kv) + 4 * rows, "flops": 10 * D * case["Hq"] * _pairs(case)}


def _exact_orth(case, st):
    a, b, c = COEFFS
    out = torch.zeros(st["update"].numel(), dtype=torch.float64, device="cuda")
    for m, n, at in st["places"]:
        g = st["update"][at:at + m * n].double().view(m, n)
        x = g / (torch.linalg.vector_norm(g) + EPS)
        for _ in range(STEPS):                                          # the small side's Gram matrix, from whichever side that is
            if m <= n:
                s = torch.mm(x, x.t())
                x = a * x + b * torch.mm(s, x) + c * torch.mm(s, torch.mm(s, x))
            else:
                s = torch.mm(x.t(), x)
                x = a * x + b * torch.mm(x, s) + c * torch.mm(torch.mm(x, s), s)
        out[at:at + m * n] = x.reshape(-1)
    return out


def _exact_rope(case, st):
    r, length = case["rot"], 4096
    x = st["x"].double()
    y = x.clone()
    pos = st["positions"].double()
    for i in range(r // 2):
        theta, gain = 10000.0 ** (-2.0 * i / r), 1.0
        if case["scaling"] == "linear":
            theta = theta / 4.0
        elif case["scaling"] == "ntk":
            theta = theta * 8.0 ** (-2.0 * i / (r - 2.0))
        elif case["scaling"] == "yarn":
            bounds = [r / 2.0 * math.log(length / (t * 2.0 * math.pi)) / math.log(10000.0) for t in (32.0, 1.0)]
            lo, hi = max(math.floor(bounds[0]), 0), min(math.ceil(bounds[1]), r - 1)
            share = min(max((i - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
            theta, gain = theta * (1.0 - share * (1.0 - 1.0 / 16.0)), 0.1 * math.log(16.0) + 1.0
        cs, sn = gain * torch.cos(pos * theta)[:, :, None], gain * torch.sin(pos * theta)[:, :, None]
        if case["inverse"]:
            sn = -sn
        p, q = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + r // 2)
        y[..., p], y[..., q] = cs * x[..., p] - sn * x[..., q], sn * x[..., p] + cs * x[..., q]
    return y


def _exact_attention(case, st):
    B, Hq, Hkv, Sq, Sk, D = (case[k] for k in ("B", "Hq", "Hkv", "Sq", "Sk", "D"))
    q, k, v, do = (st[n].double() for n in ("q", "k", "v", "dout"))
    back = case["op"] == "attn_bwd"
    o = torch.zeros_like(q)
    lse = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    rows = torch.arange(Sq, device="cuda")
    for b in range(B):
        n = int(st["lens"][b]) if case["lens"] else Sk
        if n == 0:
            continue
        hidden = torch.arange(n, device="cuda")[None] > rows[:, None] + (Sk - Sq) if case["causal"] else None
        for h in range(Hq):
            kk, vv = k[b, :n, h * Hkv // Hq], v[b, :n, h * Hkv // Hq]
            s = torch.mm(q[b, :, h], kk.t()) * D ** -0.5
            if hidden is not None:
                s[hidden] = -math.inf
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(l.isinf(), torch.zeros_like(l), l)[:, None])
            lse[b, h] = l
            if not back:
                o[b, :, h] = torch.mm(p, vv)
                continue
            g = do[b, :, h]
            ds = p * (torch.mm(g, vv.t()) - (g * st["out"][b, :, h].double()).sum(1, keepdim=True)) * D ** -0.5
            dq[b, :, h] = torch.mm(ds, kk)
            dk[b, :n, h * Hkv // Hq] += torch.mm(ds.t(), q[b, :, h])
            dv[b, :n, h * Hkv // Hq] += torch.mm(p.t(), g)
    return (dq, dk, dv) if back else (o, lse)


def exact(case, seed):
    st = prepare(case, seed)
    return {"orth": _exact_orth, "rope": _exact_rope}.get(case["op"], _exact_attention)(case, st)
