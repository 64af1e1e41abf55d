"""Norms around a block against the formulas in 64 bits.

Tolerances.  A result is computed in fp32 and rounded to its type once: half a step of its type, u = eps / 2, of the value.
The fp32 part is a few dozen operations, sums of which are chains of at most 64 with trees behind them, approximate exponentials and
square roots of 2^-21: 128 * 2^-24 = 8e-6 of the formula's value with every term taken by its magnitude.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F32 = 128 * 2.0 ** -24


def act(by, a):
    s = {None: lambda v: v, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[by](a)
    slope = {None: torch.ones_like(a), "sigmoid": s * (1 - s), "tanh": 1 - s * s}[by]
    return s, slope


def over(gate, x):
    """A gate's rows over all tokens."""
    if gate is None:
        return torch.ones((), dtype=torch.float64, device=x.device)
    g = gate.double()
    return g[:, None] if g.dim() == 2 and x.dim() == 3 else g


def plain_forward(x, f, gate, by, post, scale, pre, eps):
    """(out, normed, rows) and the magnitudes of the first two."""
    X = x.double()
    D = x.shape[-1]
    rf = rx = torch.zeros(x.shape[:-1], dtype=torch.float64, device=x.device)
    out, size = X, X.abs()
    if f is not None:
        n = f.double()
        if post is not None:
            rf = (n.square().sum(-1) / D + eps) ** -0.5
            n = n * rf[..., None] * post.double()
        add = scale * act(by, over(gate, x))[0] * n
        out, size = X + add, X.abs() + add.abs()
    normed = normed_size = None
    if pre is not None:
        rx = (out.square().sum(-1) / D + eps) ** -0.5
        normed, normed_size = out * rx[..., None] * pre.double(), size * rx[..., None] * pre.double().abs()
    return out, normed, torch.stack([rf, rx]), size, normed_size


def plain_backward(dout, dnormed, out, f, rows, gate, by, post, scale, pre):
    """The five gradients, and their magnitudes."""
    rf, rx = rows.double()[..., None].unbind(0)
    zero = torch.zeros_like(out, dtype=torch.float64)
    t = zero if dout is None else dout.double()
    size, results, sizes = t.abs(), [None] * 5, [None] * 5
    tokens = tuple(range(out.dim() - 1))
    if pre is not None:
        if dnormed is not None:
            hat, dh, w = out.double() * rx, dnormed.double(), pre.double()
            a = dh * w
            t = t + rx * (a - hat * (a * hat).mean(-1, keepdim=True))
            size = size + rx * (a.abs() + hat.abs() * (a * hat).abs().mean(-1, keepdim=True))
            results[4], sizes[4] = (dh * hat).sum(tokens), (dh * hat).abs().sum(tokens)
        else:
            results[4] = sizes[4] = torch.zeros_like(pre, dtype=torch.float64)
    results[0], sizes[0] = t, size
    if f is None:
        return results, sizes
    n = f.double() * (rf if post is not None else 1.0)
    w = 1.0 if post is None else post.double()
    g, slope = act(by, over(gate, out))
    e, e_size = scale * g * t * w, (scale * g * w).abs() * size
    results[1], sizes[1] = e, e_size
    if post is not None:
        results[1] = rf * (e - n * (e * n).mean(-1, keepdim=True))
        sizes[1] = rf * (e_size + n.abs() * (e_size * n.abs()).mean(-1, keepdim=True))
        results[3], sizes[3] = (scale * g * t * n).sum(tokens), (scale * g * size * n).abs().sum(tokens)
    if gate is not None:
        d, d_size = scale * slope * t * n * w, (scale * slope * size * n * w).abs()
        over_tokens = tokens if gate.dim() == 1 else (1,) if gate.dim() < out.dim() else ()
        results[2], sizes[2] = (d.sum(over_tokens), d_size.sum(over_tokens)) if over_tokens else (d, d_size)
    return results, sizes


def close(got, want, size, what):
    assert got.shape == want.shape, what
    if want.numel() == 0:
        return
    u = torch.finfo(got.dtype).eps / 2 if got.dtype != torch.float32 else 0.0
    least = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps          # a step among the smallest numbers of the type
    bad = (got.double() - want).abs() > u * want.abs() + F32 * size + least
    assert not bool(bad.any()), (what, float((got.double() - want).abs().max()), int(bad.sum()))


def make(shape, dtype="bf16", stream=None, gate=None, post=True, pre=True, block=True, gains="f32", wide=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, D = TYPES[dtype], shape[-1]
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    cut = lambda x: x[..., :D]  # noqa: E731
    x = cut(2 * r(*shape[:-1], D + wide)).to(TYPES[stream or dtype])
    if wide:
        x = cut(r(*shape[:-1], D + wide).to(x.dtype))
    f = cut(r(*shape[:-1], D + wide).to(t)) if block else None
    gain = lambda: (1 + 0.3 * r(D)).to(TYPES["f32"] if gains == "f32" else t)  # noqa: E731
    rows = {None: None, "channel": (D,), "sequence": (shape[0], D), "token": shape}[gate]
    return {"x": x, "f": f, "gate": None if rows is None else (0.4 + r(*rows)).to(t if gate == "token" or gains != "f32" else torch.float32),
            "post": gain() if post and block else None, "pre": gain() if pre else None,
            "dout": r(*shape).to(x.dtype), "dnormed": r(*shape).to(t if block else x.dtype) if pre else None}


def both(m, by=None, scale=0.7, eps=1e-5, dout=True, dnormed=True):
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    how = {"gate": m["gate"], "gate_by": by, "post": m["post"], "scale": scale, "pre": m["pre"], "eps": eps}
    out, normed, rows = residual_norm_forward(m["x"], m["f"], **how)
    want, want_normed, want_rows, size, normed_size = plain_forward(m["x"], m["f"], m["gate"], by, m["post"], scale, m["pre"], eps)
    if m["f"] is not None:
        close(out, want, size, "out")
    else:
        assert out is m["x"]
    assert (normed is None) == (m["pre"] is None)
    if normed is not None:
        close(normed, want_normed, normed_size, "normed")
    close(rows, want_rows, want_rows.abs() * (1 + size.amax(-1) / want.abs().amax(-1).clamp_min(1e-30)), "rows")
    dn = m["dnormed"] if dnormed else None
    got = residual_norm_backward(m["dout"] if dout else None, dn, out, m["f"], rows, **how)
    wants, sizes = plain_backward(m["dout"] if dout else None, dn, out, m["f"], rows, m["gate"], by, m["post"], scale, m["pre"])
    for name, a, b, s in zip(("dx", "df", "dgate", "dpost", "dpre"), got, wants, sizes):
        assert (a is None) == (b is None), name
        if a is not None:
            close(a, b, s, name)
    return (out, normed, rows), got


SHAPES = [(1, 1, 1), (1, 1, 8), (2, 3, 40), (3, 7, 255), (2, 33, 256), (5, 9, 257), (1, 40, 512), (2, 19, 1001), (3, 50, 1024), (2, 31, 2048), (1, 17, 4096),
          (2, 9, 4104), (1, 5, 8192), (1, 6, 8200), (1, 3, 16384), (37, 1, 96), (700, 2, 64)]


@pytest.mark.parametrize("gate, by", [(None, None), ("channel", "tanh"), ("sequence", "sigmoid"), ("token", None)])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_formula(shape, gate, by):
    both(make(shape, gate=gate, seed=shape[-1]), by)


@pytest.mark.parametrize("dtype, stream, gains", [("f32", None, "f32"), ("f16", None, "same"), ("bf16", "f32", "same"), ("f16", "f32", "f32"), ("bf16", None, "same")])
@pytest.mark.parametrize("gate, by", [("channel", None), ("sequence", "tanh"), ("token", "sigmoid")])
@pytest.mark.parametrize("D", [72, 333, 1536, 5000])
def test_types(dtype, stream, gains, gate, by, D):
    both(make((3, 29, D), dtype, stream, gate, gains=gains), by)


@pytest.mark.parametrize("post, pre, block", [(True, False, True), (False, True, True), (False, False, True), (False, True, False)])
@pytest.mark.parametrize("gate", [None, "channel", "token"])
@pytest.mark.parametrize("D", [64, 4096, 77])
def test_parts_left_out(post, pre, block, gate, D):
    both(make((2, 21, D), gate=gate if block else None, post=post, pre=pre, block=block))


def test_gradients_that_are_not_there():
    m = make((2, 30, 520), gate="sequence")
    both(m, dout=False)
    both(m, dnormed=False)


@pytest.mark.parametrize("wide", [8, 24, 5])
def test_slices_of_wider_rows_and_two_dimensions(wide):
    m = make((3, 25, 248), gate="token", wide=wide)
    both(m)
    flat = {k: None if v is None else v.flatten(0, 1) if v.dim() == 3 else v for k, v in m.items()}
    both(flat)
    odd = {k: v if v is None or v.dim() != 3 else torch.cat([v.flatten()[:1], v.flatten()])[1:].view(v.shape) for k, v in m.items()}     # off every boundary
    both(odd)


@pytest.mark.parametrize("dtype, gate", [("bf16", "token"), ("f32", "token"), ("f16", "sequence")])
@pytest.mark.parametrize("D", [8, 264, 520, 1000, 4096, 8184])
def test_fp32_rows_on_16_bytes(D, dtype, gate):
    """Rows of an fp32 stream that start on 16 bytes but not on 32 and end inside what a warp moves at once; results there too, the same bits, nothing around them touched."""
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    m = make((3, 167, D), dtype, "f32", gate)

    def moved(t, fill=None):
        if t is None or t.dim() != 3 or t.dtype != torch.float32:
            return t
        room = torch.full((*t.shape[:-1], D + 12), 7.0, device="cuda")
        room[..., 4:-8] = t if fill is None else fill
        return room[..., 4:-8]

    a, b = both(m, "tanh"), both({k: moved(v) for k, v in m.items()}, "tanh")
    for one, two in zip((*a[0], *a[1]), (*b[0], *b[1])):
        assert torch.equal(one, two)
    how = {"gate": m["gate"], "gate_by": "tanh", "post": m["post"], "scale": 0.7, "pre": m["pre"], "eps": 1e-5}
    to = [moved(t, 0.0) for t in (a[0][0], a[1][0])]
    residual_norm_forward(m["x"], m["f"], out=to[0], **how)
    residual_norm_backward(m["dout"], m["dnormed"], a[0][0], m["f"], a[0][2], dx=to[1], **how)
    for t, want in zip(to, (a[0][0], a[1][0])):
        assert torch.equal(t, want)
        room = t._base
        assert bool((room[..., :4] == 7).all()) and bool((room[..., -8:] == 7).all())


def test_time_first_memory():
    m = make((4, 50, 136), gate="sequence")
    turned = {k: v.transpose(0, 1).contiguous().transpose(0, 1) if v is not None and v.dim() == 3 else v for k, v in m.items()}
    a, b = both(m), both(turned)
    for one, two in zip((*a[0], *a[1]), (*b[0], *b[1])):
        assert torch.equal(one, two)


@pytest.mark.parametrize("shape", [(4, 2000, 1024), (1, 3000, 4096), (64, 100, 333)])
def test_many_tokens_and_repeats(shape):
    """More rows than run at once; the same bits every time."""
    m = make(shape, "bf16", "f32", "sequence")
    first = both(m, "sigmoid")
    for _ in range(3):
        again = both(m, "sigmoid")
        for one, two in zip((*first[0], *first[1]), (*again[0], *again[1])):
            assert torch.equal(one, two)


def test_no_tokens():
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    for shape in ((0, 5, 64), (3, 0, 64)):
        m = make(shape, gate="sequence")
        how = {k: m[k] for k in ("gate", "post", "pre")}
        out, normed, rows = residual_norm_forward(m["x"], m["f"], **how)
        assert out.shape == normed.shape == shape and rows.shape == (2, *shape[:2])
        dx, df, dgate, dpost, dpre = residual_norm_backward(m["dout"], m["dnormed"], out, m["f"], rows, **how)
        assert dx.shape == df.shape == shape and dgate.shape == (shape[0], 64)
        assert not dgate.any() and not dpost.any() and not dpre.any()


def test_rows_of_zeros_infinities_and_nan_stay_by_themselves():
    from paper_2411_03742_b200 import residual_norm_forward
    m = make((1, 40, 512))
    clean = residual_norm_forward(m["x"], m["f"], post=m["post"], pre=m["pre"])
    x, f = m["x"].clone(), m["f"].clone()
    x[0, 3], f[0, 5, 7], x[0, 9, 0] = 0.0, float("nan"), float("inf")
    f[0, 3] = 0.0
    out, normed, rows = residual_norm_forward(x, f, post=m["post"], pre=m["pre"])
    keep = [i for i in range(40) if i not in (3, 5, 9)]
    for a, b in zip((out, normed), clean):
        assert torch.equal(a[0, keep], b[0, keep])
    assert torch.equal(rows[:, 0, keep], clean[2][:, 0, keep])
    assert not out[0, 3].any() and not normed[0, 3].any() and out[0, 5].isnan().all() and normed[0, 5].isnan().all() and normed[0, 9].isnan().any()


def test_in_place():
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    m = make((2, 100, 640), gate="token")
    how = {"gate": m["gate"], "gate_by": "tanh", "post": m["post"], "pre": m["pre"]}
    out, normed, rows = residual_norm_forward(m["x"], m["f"], **how)
    x = m["x"].clone()
    again = residual_norm_forward(x, m["f"], out=x, **how)
    assert again[0] is x and torch.equal(x, out) and torch.equal(again[1], normed) and torch.equal(again[2], rows)
    want = residual_norm_backward(m["dout"], m["dnormed"], out, m["f"], rows, **how)
    dout = m["dout"].clone()
    got = residual_norm_backward(dout, m["dnormed"], out, m["f"], rows, dx=dout, **how)
    assert got[0] is dout and all(torch.equal(a, b) for a, b in zip(got, want))


def test_autograd_against_the_formula():
    """residual_norm's gradients against autograd through the same formula in 64 bits, gates broadcast and expanded."""
    from paper_2411_03742_b200 import residual_norm
    for gate_shape in ((48,), (3, 48), (3, 20, 48), "expanded"):
        m = make((3, 20, 48), "f32")
        gate = torch.randn((3, 20, 48) if gate_shape == "expanded" else gate_shape, device="cuda")
        if gate_shape == "expanded":
            gate = gate[:, :1].expand(3, 20, 48)
        leaves = [t.clone().requires_grad_() for t in (m["x"], m["f"], m["post"], m["pre"])] + [gate.detach().requires_grad_()]
        x, f, post, pre, g = leaves
        out, normed = residual_norm(x, f, gate=g, gate_by="sigmoid", post=post, pre=pre, scale=0.5)
        got = torch.autograd.grad((out * m["dout"]).sum() + (normed * m["dnormed"]).sum(), leaves)
        wide = [t.detach().double().requires_grad_() for t in leaves]
        X, F, P, Q, G = wide
        n = F / (F.square().mean(-1, keepdim=True) + 1e-6).sqrt() * P
        new = X + 0.5 * torch.sigmoid(G[:, None] if G.dim() == 2 else G) * n
        h = new / (new.square().mean(-1, keepdim=True) + 1e-6).sqrt() * Q
        want = torch.autograd.grad((new * m["dout"].double()).sum() + (h * m["dnormed"].double()).sum(), wide)
        for a, b in zip(got, want):
            assert float((a.double() - b).norm() / b.norm()) <= 1e-5


def test_gradient_against_differences():
    """Along a random direction the loss changes by the gradient's product with it: central differences in 64 bits of the plain form."""
    from paper_2411_03742_b200 import residual_norm
    m = make((2, 9, 40), "f32", gate="sequence")
    leaves = [m[k].clone().requires_grad_() for k in ("x", "f", "gate", "post", "pre")]
    x, f, gate, post, pre = leaves
    out, normed = residual_norm(x, f, gate=gate, gate_by="tanh", post=post, pre=pre, scale=0.7, eps=1e-5)
    grads = torch.autograd.grad((out * m["dout"]).sum() + (normed * m["dnormed"]).sum(), leaves)

    def loss(values):
        o, h, *_ = plain_forward(values[0], values[1], values[2], "tanh", values[3], 0.7, values[4], 1e-5)
        return float((o * m["dout"].double()).sum() + (h * m["dnormed"].double()).sum())

    for k, g in enumerate(grads):
        d = torch.randn_like(g).double()
        step = 1e-5
        up, down = ([v.detach().double() + (s * step * d if i == k else 0) for i, v in enumerate(leaves)] for s in (1, -1))
        want = (loss(up) - loss(down)) / (2 * step)
        # the differences are good to step^2 times a third derivative, the gradient to F32 of its size
        assert abs(float((g.double() * d).sum()) - want) <= 1e-4 * float((g.double().abs() * d.abs()).sum())


def test_part_of_the_graph():
    """Only one of the results used; no gradient asked for x or the gains; a frozen block."""
    from paper_2411_03742_b200 import residual_norm
    m = make((2, 12, 64), "f32")
    x, f, pre = (m[k].clone().requires_grad_() for k in ("x", "f", "pre"))
    for pick in (0, 1):
        r = residual_norm(x, f.detach() if pick else f, post=m["post"], pre=pre if pick else None)
        g = torch.autograd.grad(r[pick].sum(), [x] if pick else [x, f])
        assert all(t is not None and bool(t.isfinite().all()) for t in g)
    out, normed = residual_norm(x, pre=pre)
    assert out is x
    gx, gp = torch.autograd.grad(normed.square().sum(), (x, pre))
    X, P = x.detach().double().requires_grad_(), pre.detach().double().requires_grad_()
    want = torch.autograd.grad((X / (X.square().mean(-1, keepdim=True) + 1e-6).sqrt() * P).square().sum(), (X, P))
    assert all(float((a.double() - b).norm() / b.norm()) <= 1e-5 for a, b in zip((gx, gp), want))
    with pytest.raises(NotImplementedError, match="once"):
        one, = torch.autograd.grad(residual_norm(x, pre=pre)[1].square().sum(), x, create_graph=True)
        torch.autograd.grad(one.sum(), x)


def test_replayed_from_a_graph_and_on_another_stream():
    from paper_2411_03742_b200 import residual_norm_backward, residual_norm_forward
    m = make((3, 200, 1024), "bf16", "f32", "channel")
    how = {"gate": m["gate"], "gate_by": "sigmoid", "post": m["post"], "pre": m["pre"]}

    def step():
        made = residual_norm_forward(m["x"], m["f"], **how)
        return (*made, *residual_norm_backward(m["dout"], m["dnormed"], made[0], m["f"], made[2], **how))

    want = [t.clone() for t in step()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    keep = m["x"].clone()
    m["x"].zero_()
    g.replay()
    m["x"].copy_(keep)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    made = residual_norm_forward(m["x"], m["f"], stream=side, **how)
    back = residual_norm_backward(m["dout"], m["dnormed"], made[0], m["f"], made[2], stream=side, **how)
    rubbish = [torch.full((3 * 200 * 1024,), float("nan"), device="cuda") for _ in range(6)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((*made, *back), want))
    del rubbish


def test_far_offsets():
    """Rows beyond 2^31 elements from the tensor's start."""
    from paper_2411_03742_b200 import residual_norm_forward
    big = torch.empty(2 ** 31 + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(big, (2, 3, 256), (2 ** 31, 1024, 1))
    x.copy_(torch.randn((2, 3, 256), device="cuda"))
    f, pre = torch.randn((2, 3, 256), device="cuda").bfloat16(), torch.ones(256, device="cuda")
    a, b = residual_norm_forward(x, f, pre=pre), residual_norm_forward(x.contiguous(), f, pre=pre)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
