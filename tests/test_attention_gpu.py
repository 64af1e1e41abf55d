"""Attention and its gradient against the formulas in 64 bits.

Tolerances.  u = 2^-8 (bf16) or 2^-11 (fp16) is the largest relative rounding error of the type, 0.43 u its rms.
An output is a sum whose terms each carry one rounding (of P or dS) and is rounded itself: independent
errors of 0.43 u each, 0.6 u of the output's norm together; u is allowed.  A single element may lie 4 u of
itself plus 8 u of the tensor's rms off.  lse: S and the sums are fp32, 1e-5 absolute.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def heads(x, groups=1):
    return x.double().transpose(1, 2).repeat_interleave(groups, 1)


def plain_forward(q, k, v, scale, causal, lens):
    """O, lse and P in 64 bits (head-major)."""
    r = q.shape[2] // k.shape[2]
    Sq, Sk = q.shape[1], k.shape[1]
    s = heads(q) @ heads(k, r).mT * scale
    j, i = torch.arange(Sk, device=q.device), torch.arange(Sq, device=q.device)[:, None]
    hidden = torch.zeros((q.shape[0], 1, Sq, Sk), dtype=torch.bool, device=q.device)
    if lens is not None:
        hidden = hidden | (j >= lens[:, None])[:, None, None]
    if causal:
        hidden = hidden | (j > i + Sk - Sq)
    s = s.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.clamp_min(-1e300)[..., None]).masked_fill(hidden, 0.0)
    return p @ heads(v, r), lse, p


def plain_backward(q, k, v, scale, p, out, dout):
    B, Sq, Hq, D = q.shape
    Sk, Hk = k.shape[1:3]
    r = Hq // Hk
    dp = heads(dout) @ heads(v, r).mT
    ds = p * (dp - (heads(dout) * heads(out)).sum(-1, keepdim=True)) * scale
    share = lambda x: x.view(B, Hk, r, Sk, D).sum(2)  # noqa: E731
    return ds @ heads(k, r), share(ds.mT @ heads(q)), share(p.mT @ heads(dout))


def close(got, want, dtype, what):
    got = got.double().transpose(1, 2)
    assert got.shape == want.shape
    if want.numel() == 0:
        return
    diff, u = (got - want).abs(), U[dtype]
    norm, rms = float(want.norm()), float(want.norm()) / math.sqrt(want.numel())
    assert float(diff.norm()) <= u * norm + 1e-30, (what, float(diff.norm()) / max(norm, 1e-30))
    assert bool((diff <= 4 * u * want.abs() + 8 * u * rms + 1e-30).all()), (what, float(diff.max()), rms)


def check(B, Sq, Sk, Hq, Hk, D, causal=False, lens=None, dtype=torch.bfloat16, packed=False, scale=None, seed=0, poison=False, heads_first=False):
    from paper_2411_03742_b200 import attention, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    if packed:
        x = rnd(B, Sq, Hq + 2 * Hk, D)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hk], x[:, :, Hq + Hk:]
    else:
        q, k, v = rnd(B, Sq, Hq, D), rnd(B, Sk, Hk, D), rnd(B, Sk, Hk, D)
    if heads_first:
        q, k, v = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v))
    dout = rnd(B, Sq, Hq, D)
    L = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    ks, vs = k, v
    if poison:                                        # what lies past a batch's keys is nobody's business
        k, v = k.clone(), v.clone()
        for b, n in enumerate(lens):
            k[b, n:], v[b, n:] = math.nan, math.inf
    sc = 1 / math.sqrt(D) if scale is None else scale
    out, lse = attention_forward(q, k, v, scale=scale, causal=causal, kv_lens=L)
    grads = attention_backward(dout, q, k, v, out, lse, scale=scale, causal=causal, kv_lens=L)
    torch.cuda.synchronize()
    assert attention.status() == 0
    O, LSE, P = plain_forward(q, ks, vs, sc, causal, L)
    close(out, O, dtype, "out")
    none = LSE == -math.inf
    assert torch.equal(lse == -math.inf, none)
    assert float((lse.double() - LSE).masked_fill(none, 0.0).abs().max()) <= 1e-5
    assert not out.transpose(1, 2)[none].any(), "a query without keys has a zero output"
    for name, got, want in zip(("dq", "dk", "dv"), grads, plain_backward(q, ks, vs, sc, P, out, dout)):
        close(got, want, dtype, name)
    if lens is not None:
        for b, n in enumerate(lens):
            assert not grads[1][b, n:].any() and not grads[2][b, n:].any(), "gradients of hidden keys are zero"
    return out, lse, grads


@pytest.mark.parametrize("D", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("Sq, Sk", [(16, 16), (128, 128), (129, 127), (256, 256), (257, 255), (300, 700), (77, 91)])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_and_head_sizes(D, Sq, Sk, causal):
    check(2, Sq, Sk, 2, 2, D, causal)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq, Hk", [(1, 1), (4, 2), (6, 1), (8, 8)])
def test_shared_heads(dtype, Hq, Hk):
    check(2, 200, 330, Hq, Hk, 64, True, dtype=dtype)
    check(1, 140, 140, Hq, Hk, 128, False, dtype=dtype, packed=True)


def test_single_tokens_over_long_keys():
    check(3, 1, 1000, 4, 2, 128, True)
    check(2, 1, 4097, 2, 2, 64, False, lens=[4097, 3])
    check(1, 2, 129, 1, 1, 80, True)


def test_queries_before_the_first_key():
    """Causal with more queries than keys: the first rows see nothing."""
    check(2, 391, 100, 4, 1, 128, True)
    check(1, 700, 20, 2, 2, 64, True)


@pytest.mark.parametrize("lens", [[0, 0, 0], [1, 0, 333], [333, 128, 127], [129, 256, 255]])
@pytest.mark.parametrize("causal", [False, True])
def test_padded_batches_with_rubbish_behind_them(lens, causal):
    check(3, 333, 333, 4, 2, 64, causal, lens=lens, poison=True)
    check(3, 150, 333, 2, 1, 128, causal, lens=lens, poison=True)


def test_lengths_out_of_range_are_clamped():
    from paper_2411_03742_b200 import attention_forward
    q = torch.randn((2, 30, 2, 64), device="cuda").bfloat16()
    a = attention_forward(q, q, q, kv_lens=torch.tensor([-5, 1000], dtype=torch.int32, device="cuda"))
    b = attention_forward(q, q, q, kv_lens=torch.tensor([0, 30], dtype=torch.int32, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_empty_tensors():
    from paper_2411_03742_b200 import attention_backward, attention_forward
    z = lambda *s: torch.ones(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    out, lse = attention_forward(z(2, 5, 2, 64), z(2, 0, 2, 64), z(2, 0, 2, 64))
    assert not out.any() and (lse == -math.inf).all()
    dq, dk, dv = attention_backward(z(2, 5, 2, 64), z(2, 5, 2, 64), z(2, 0, 2, 64), z(2, 0, 2, 64), out, lse)
    assert not dq.any() and dk.shape == (2, 0, 2, 64)
    out, lse = attention_forward(z(2, 0, 2, 64), z(2, 7, 2, 64), z(2, 7, 2, 64))
    assert out.shape == (2, 0, 2, 64)
    dq, dk, dv = attention_backward(z(2, 0, 2, 64), z(2, 0, 2, 64), z(2, 7, 2, 64), z(2, 7, 2, 64), out, lse)
    assert not dk.any() and not dv.any()
    out, lse = attention_forward(z(0, 4, 2, 64), z(0, 7, 2, 64), z(0, 7, 2, 64))
    assert out.numel() == 0


def test_large_scores_and_growing_maxima():
    """Scores of several hundred, and keys whose scores grow along the sequence: the maximum moves at every tile."""
    from paper_2411_03742_b200 import attention_forward
    check(1, 200, 900, 2, 1, 64, scale=8.0 / 8)
    q = torch.ones((1, 130, 1, 64), device="cuda").bfloat16()
    k = (torch.arange(1200, device="cuda").float()[None, :, None, None] / 16).expand(1, 1200, 1, 64).bfloat16().contiguous()
    v = torch.randn((1, 1200, 1, 64), device="cuda").bfloat16()
    out, lse = attention_forward(q, k, v)
    O, LSE, _ = plain_forward(q, k, v, 0.125, False, None)
    close(out, O, torch.bfloat16, "out")
    assert float((lse.double() - LSE).abs().max()) <= 1e-6 * float(LSE.abs().max())
    out, lse = attention_forward(q, k.flip(1).contiguous(), v)
    O, LSE, _ = plain_forward(q, k.flip(1), v, 0.125, False, None)
    close(out, O, torch.bfloat16, "out")


def test_memory_orders():
    a = check(2, 150, 150, 4, 2, 64, True, packed=True)
    b = check(2, 150, 150, 4, 2, 64, True, packed=True, heads_first=True)
    for x, y in zip((a[0], a[1], *a[2]), (b[0], b[1], *b[2])):
        assert torch.equal(x, y)


def test_given_outputs_streams_and_repeats():
    """Results written into slices of larger buffers, on another stream, again: the same bytes, and nothing beside them."""
    from paper_2411_03742_b200 import attention_backward, attention_forward
    from paper_2411_03742_b200.attention import workspace_bytes
    B, S, H, D = 2, 333, 4, 72
    q, k, v, dout = (torch.randn((B, S, H, D), device="cuda").bfloat16() for _ in range(4))
    out, lse = attention_forward(q, k, v, causal=True)
    grads = attention_backward(dout, q, k, v, out, lse, causal=True)
    big = torch.full((4, B, S + 3, H + 2, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    places = [t[:, 1:S + 1, 1:H + 1, :D] for t in big]
    work = torch.full((workspace_bytes(q, k),), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    l2 = torch.empty_like(lse)
    attention_forward(q, k, v, causal=True, out=places[0], lse=l2, stream=side)
    attention_backward(dout, q, k, v, places[0], l2, causal=True, dq=places[1], dk=places[2], dv=places[3], workspace=work, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(l2, lse)
    for got, want in zip(places, (out, *grads)):
        assert torch.equal(got, want)
    for t, place in zip(big, places):
        inside = int(place.numel())
        assert int((t == 7.0).sum()) >= t.numel() - inside
        assert (t[:, 0] == 7.0).all() and (t[:, S + 1:] == 7.0).all() and (t[..., D:] == 7.0).all()


@pytest.mark.parametrize("B, Sq, Sk, Hq, Hk, D, causal, lens", [
    (1, 1, 4000, 4, 1, 128, False, None), (3, 1, 1111, 2, 2, 64, True, [1111, 0, 300]), (1, 200, 3000, 4, 2, 72, True, None), (2, 130, 2049, 2, 1, 40, False, [1, 2049]),
    (1, 3000, 3000, 2, 1, 64, True, None), (1, 700, 500, 2, 1, 128, True, None), (2, 257, 1500, 1, 1, 96, False, [129, 700])])
def test_few_rows_over_many_keys(B, Sq, Sk, Hq, Hk, D, causal, lens):
    """Several blocks share a tile's walk over the other side, some of them without anything to see.  Rows of dk and dv are as
    large as their keys' probabilities, which differ by orders here, so each element's bound is u times the sum of its terms' sizes:
    one unit for P or dS (rounded to 16 bits, half a unit), for Delta (from the rounded out), and for the result itself."""
    from paper_2411_03742_b200 import attention, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sq + Sk)
    q, dout = (torch.randn((B, Sq, Hq, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((B, Sk, Hk, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    L = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = attention_forward(q, k, v, causal=causal, kv_lens=L)
    grads = attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=L)
    again = attention_forward(q, k, v, causal=causal, kv_lens=L) + attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=L)
    torch.cuda.synchronize()
    assert attention.status() == 0
    assert all(torch.equal(x, y) for x, y in zip((out, lse) + grads, again)), "shares are joined in one order"
    sc, r, u = 1 / math.sqrt(D), Hq // Hk, U[torch.bfloat16]
    O, LSE, P = plain_forward(q, k, v, sc, causal, L)
    none = LSE == -math.inf
    assert torch.equal(lse == -math.inf, none) and float((lse.double() - LSE).masked_fill(none, 0.0).abs().max()) <= 1e-5
    K, V, dO = heads(k, r), heads(v, r), heads(dout)
    dq, dk, dv = plain_backward(q, k, v, sc, P, out, dout)
    ds = P * (dO @ V.mT - (dO * heads(out)).sum(-1, keepdim=True)) * sc
    slack = ds.abs() + P * (dO * heads(out)).abs().sum(-1, keepdim=True) * sc
    share = lambda x: x.view(B, Hk, r, Sk, D).sum(2)  # noqa: E731
    for name, got, want, terms in (("out", out, O, P @ V.abs()), ("dq", grads[0], dq, slack @ K.abs()), ("dk", grads[1], dk, share(slack.mT @ heads(q).abs())),
                                   ("dv", grads[2], dv, share(P.mT @ dO.abs()))):
        err = (got.double().transpose(1, 2) - want).abs()
        assert bool((err <= u * (terms + want.abs()) + 1e-30).all()), (name, float((err - u * (terms + want.abs())).max()))


@pytest.mark.parametrize("B, Sq, Sk, Hq, Hk, D, causal", [(3, 77, 91, 4, 2, 40, False), (1, 1, 300, 2, 1, 128, True), (2, 128, 129, 4, 2, 128, False),
                                                           (1, 256, 256, 3, 3, 64, True), (2, 65, 1, 2, 2, 72, False)])
def test_short_queries_with_and_without_a_workspace(B, Sq, Sk, Hq, Hk, D, causal):
    """The statistics made in each block and those of the kernel before it are the same sums: the gradients agree bit for bit."""
    from paper_2411_03742_b200 import attention_backward, attention_forward
    from paper_2411_03742_b200.attention import workspace_bytes
    g = torch.Generator(device="cuda").manual_seed(Sq + D)
    q, dout = (torch.randn((B, Sq, Hq, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((B, Sk, Hk, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    lens = torch.randint(0, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    out, lse = attention_forward(q, k, v, causal=causal, kv_lens=lens)
    work = torch.full((workspace_bytes(q, k),), 255, dtype=torch.uint8, device="cuda")
    one = attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=lens)
    two = attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=lens, workspace=work)
    assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_long_queries_need_a_workspace():
    import ctypes
    from paper_2411_03742_b200.attention import SHORT_ROWS, _Shape, _Tensor
    from paper_2411_03742_b200.binding import EINVAL, load_library
    for q_len, q_heads in ((SHORT_ROWS + 1, 1), (1, SHORT_ROWS // 128 + 1)):
        t = torch.zeros((1, q_len, q_heads, 64), dtype=torch.bfloat16, device="cuda")
        rows = torch.zeros((1, q_heads, q_len), device="cuda")
        s, x = _Shape(1, 1, q_heads, 1, q_len, q_len, 64, 0, 0.125, None), _Tensor(t.data_ptr(), *t.stride()[:3])
        r = ctypes.byref
        assert load_library().adacons_attn_backward(r(s), r(x), r(x), r(x), r(x), r(x), rows.data_ptr(), r(x), r(x), r(x), None, 0, None) == EINVAL


def test_strides_past_32_bits():
    from paper_2411_03742_b200 import attention_backward, attention_forward
    far = torch.zeros((1 << 31) + 64 * 140 * 2, dtype=torch.bfloat16, device="cuda")
    src = torch.randn((2, 140, 2, 64), device="cuda").bfloat16()
    q = far.as_strided((2, 140, 2, 64), (1 << 31, 128, 64, 1))
    q.copy_(src)
    out, lse = attention_forward(q, q, q)
    want, lse2 = attention_forward(src, src, src)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    for a, b in zip(attention_backward(src, q, q, q, out, lse), attention_backward(src, src, src, src, out, lse)):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    """Central differences of the 64-bit forward pass along random directions, through the differentiable call."""
    from paper_2411_03742_b200.attention import attention
    g = torch.Generator(device="cuda").manual_seed(5)
    x = [torch.randn(s, generator=g, device="cuda").half().requires_grad_() for s in ((2, 90, 4, 64), (2, 130, 2, 64), (2, 130, 2, 64))]
    lens = torch.tensor([130, 60], dtype=torch.int32, device="cuda")
    w = torch.randn((2, 90, 4, 64), generator=g, device="cuda").half()
    (attention(*x, causal=True, kv_lens=lens) * w).sum().backward()
    h = 1e-4
    for k in range(3):
        d = torch.randn(x[k].shape, generator=g, device="cuda", dtype=torch.float64)
        sides = []
        for sign in (1, -1):
            y = [t.detach().double() for t in x]
            y[k] = y[k] + sign * h * d
            sides.append(float((plain_forward(*y, 0.125, True, lens)[0].transpose(1, 2) * w.double()).sum()))
        slope = (sides[0] - sides[1]) / (2 * h)
        got = float((x[k].grad.double() * d).sum())
        # the gradient's relative error of u, seen along one direction
        assert abs(got - slope) <= 4 * U[torch.float16] * float(x[k].grad.double().norm()) * 3, (k, got, slope)


def test_broadcast_gradient_of_a_sum():
    from paper_2411_03742_b200.attention import attention
    x = [torch.randn((1, 64, 2, 64), device="cuda").bfloat16().requires_grad_() for _ in range(3)]
    attention(*x).sum().backward()
    a = [t.grad.clone() for t in x]
    for t in x:
        t.grad = None
    (attention(*x) * torch.ones((1, 64, 2, 64), dtype=torch.bfloat16, device="cuda")).sum().backward()
    for t, want in zip(x, a):
        assert torch.equal(t.grad, want)


def test_captured_in_a_graph():
    from paper_2411_03742_b200 import attention_backward, attention_forward
    q = torch.randn((2, 200, 4, 64), device="cuda").bfloat16()
    out, lse = attention_forward(q, q, q, causal=True)
    want = attention_backward(q, q, q, q, out, lse, causal=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o2, l2 = attention_forward(q, q, q, causal=True)
        got = attention_backward(q, q, q, q, o2, l2, causal=True)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o2, out) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    from paper_2411_03742_b200 import AdaConsError, attention_backward, attention_forward
    q = torch.zeros((1, 8, 2, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q[0], q.cpu(), q[..., ::2], q[..., :12], torch.zeros((1, 8, 3, 64), dtype=torch.bfloat16, device="cuda")):
        with pytest.raises(ValueError):
            attention_forward(q, bad, bad)
    with pytest.raises(ValueError):
        attention_forward(q, q, q, kv_lens=torch.zeros(1, device="cuda"))
    off = torch.zeros(1 * 8 * 2 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(1, 8, 2, 64)
    with pytest.raises(AdaConsError):                       # 8 bytes off a 16-byte boundary
        attention_forward(off, q, q)
    with pytest.raises(AdaConsError):
        attention_forward(q, q, q, scale=0.0)
    out, lse = attention_forward(q, q, q)
    with pytest.raises(AdaConsError):
        attention_backward(q, q, q, q, out, lse, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        attention_backward(q, q, q, q, out, lse.bfloat16())


def test_second_derivatives_are_refused():
    from paper_2411_03742_b200.attention import attention
    x = torch.randn((1, 64, 2, 64), device="cuda").bfloat16().requires_grad_()
    y = torch.randn((1, 64, 2, 64), device="cuda").bfloat16().requires_grad_()
    for f in (lambda: attention(x * x, x, y).float().square().sum(), lambda: attention(x * x, x, y).sum()):
        g = torch.autograd.grad(f(), x, create_graph=True)[0]
        with pytest.raises(NotImplementedError, match="once"):
            torch.autograd.grad(g.float().square().sum(), x)
    (z,) = torch.autograd.grad((attention(x, x, x) * y).sum() + (y * y * y).float().sum(), y, create_graph=True)       # what does not pass it is served
    assert torch.autograd.grad(z.float().sum(), y, allow_unused=True)[0] is not None


def test_gradients_off_a_16_byte_boundary():
    from paper_2411_03742_b200.attention import attention
    x = [torch.randn((2, 64, 2, 64), device="cuda").bfloat16().requires_grad_() for _ in range(3)]
    w = torch.randn((2 * 64 * 2 * 64 + 3,), device="cuda").bfloat16()
    a = torch.autograd.grad((torch.cat([w[:3], attention(*x).flatten()]) * w).sum(), x)
    b = torch.autograd.grad((attention(*x) * w[3:].view(2, 64, 2, 64).clone()).sum(), x)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("Sq, Sk", [(1, 4000), (130, 2049), (300, 300)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_query_with_a_nan_shows_it(Sq, Sk, D):
    """One element of one query is NaN: its row of out and lse is NaN and no other, whether its keys are shared between blocks or not;
    so are its dq and, through dS and P, the gradients of its head's keys."""
    from paper_2411_03742_b200 import attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sq)
    q, dout = (torch.randn((2, Sq, 2, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((2, Sk, 2, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    clean = attention_forward(q, k, v)
    row = Sq // 2
    q[1, row, 0, 3] = math.nan
    out, lse = attention_forward(q, k, v)
    hit = torch.zeros((2, Sq, 2), dtype=torch.bool, device="cuda")
    hit[1, row, 0] = True
    assert out[hit].isnan().all() and lse.transpose(1, 2)[hit].isnan().all()
    assert torch.equal(out[~hit], clean[0][~hit]) and torch.equal(lse.transpose(1, 2)[~hit], clean[1].transpose(1, 2)[~hit])
    dq, dk, dv = attention_backward(dout, q, k, v, out, lse)
    assert dq[hit].isnan().all() and not dq[~hit].isnan().any()
    for t in (dk, dv):
        assert t[1, :, 0].isnan().all() and not t[0].isnan().any() and not t[1, :, 1].isnan().any()
    k[0, Sk - 1, 1, 0] = math.nan                     # a key that every query sees
    out, lse = attention_forward(q, k, v)
    assert out[0, :, 1].isnan().all() and lse[0, 1].isnan().all() and not out[0, :, 0].isnan().any()


@pytest.mark.parametrize("Sq, Sk, D, H", [(200, 100, 64, 1), (200, 100, 128, 1), (700, 20, 72, 1), (391, 100, 128, 3), (3000, 500, 64, 2), (330, 300, 40, 1), (100, 37, 128, 2)])
def test_rubbish_in_queries_without_keys(Sq, Sk, D, H):
    """q and dout of the queries before the first key hold NaN and Inf: not one byte of any result changes."""
    from paper_2411_03742_b200 import attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sq)
    q, dout = (torch.randn((2, Sq, 2 * H, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn((2, Sk, 2, D), generator=g, device="cuda").bfloat16() for _ in range(2))
    results = []
    for _ in range(2):
        out, lse = attention_forward(q, k, v, causal=True)
        results.append((out, lse, *attention_backward(dout, q, k, v, out, lse, causal=True)))
        q[:, :Sq - Sk], dout[:, :Sq - Sk] = math.nan, math.inf
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert not results[1][2][:, :Sq - Sk].any()


@pytest.mark.parametrize("Sq, Sk, Hq, Hk, D, by_dout, by_v, by_qk, lens", [
    (130, 40000, 2, 1, 64, 1.0, 1.0, 1.0, None), (300, 70001, 1, 1, 128, 0.02, 1.0, 1.0, None), (1, 66000, 4, 2, 72, 1.0, 1.0, 1.0, None),
    (700, 9000, 2, 2, 40, 0.01, 0.5, 1.0, [8000, 9000]), (2000, 2000, 4, 2, 64, 1e-3, 4.0, 1.0, None), (77, 3, 2, 1, 64, 1000.0, 30.0, 0.05, None),
    (1000, 2, 1, 1, 128, 2000.0, 20.0, 0.02, [2, 1])])
def test_half_precision_far_from_one(Sq, Sk, Hq, Hk, D, by_dout, by_v, by_qk, lens):
    """fp16 gradients where P or dS would leave the type's range if they were rounded as they are: below 2^-14 on long rows and under
    small dout, above 65504 under a large one.  The bounds are those of `close`, and half a unit of the smallest fp16 numbers, 2^-25, for
    each result below 2^-14, and for dP - Delta, which a query with one key cancels to nothing, 2^-20 of the sums that are
    subtracted (fp32, which the tensor cores round toward zero).  In the last case some of dv are beyond 65504.  Values hidden behind kv_lens are Inf and must not count."""
    from paper_2411_03742_b200 import attention, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sk)
    rnd = lambda n, s, h, by: (torch.randn((n, s, h, D), generator=g, device="cuda") * by).half()  # noqa: E731
    B = 1 if lens is None else len(lens)
    q, k, v, dout = rnd(B, Sq, Hq, by_qk), rnd(B, Sk, Hk, by_qk), rnd(B, Sk, Hk, by_v), rnd(B, Sq, Hq, by_dout)
    L = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    vs = v.clone()
    for b, n in enumerate(lens or []):
        v[b, n:] = math.inf
    out, lse = attention_forward(q, k, v, kv_lens=L)
    grads = attention_backward(dout, q, k, v, out, lse, kv_lens=L)
    again = attention_backward(dout, q, k, v, out, lse, kv_lens=L)
    torch.cuda.synchronize()
    assert attention.status() == 0 and all(torch.equal(a, b) for a, b in zip(grads, again))
    sc, u, tiny = 1 / math.sqrt(D), U[torch.float16], 2.0 ** -25
    for b in range(B):                                  # one batch at a time: the 64-bit form is large
        one = slice(b, b + 1)
        _, _, P = plain_forward(q[one], k[one], vs[one], sc, False, None if L is None else L[one])
        wants = plain_backward(q[one], k[one], vs[one], sc, P, out[one], dout[one])
        r = Hq // Hk
        share = lambda x: x.view(1, Hk, r, Sk, D).sum(2)  # noqa: E731
        dO, O = heads(dout[one]).abs(), heads(out[one]).abs()
        noise = 2.0 ** -20 * sc * P * (dO @ heads(vs[one], r).abs().mT + (dO * O).sum(-1, keepdim=True))
        noises = (noise @ heads(k[one], r).abs(), share(noise.mT @ heads(q[one]).abs()), 2.0 ** -20 * share(P.mT @ dO))
        for name, got, want, extra in zip(("dq", "dk", "dv"), grads, wants, noises):
            err, n = (got[one].double().transpose(1, 2) - want).abs(), want.numel()
            beyond = want.abs() > 65504 * (1 - 4 * u)           # the type has no number for it: Inf is the answer
            assert not (err.isinf() & ~beyond).any()
            err = err.masked_fill(err.isinf() & beyond, 0.0)
            rms = float(want.norm()) / math.sqrt(n)
            assert float(err.norm()) <= u * float(want.norm()) + tiny * math.sqrt(n) + float(extra.norm()), (name, float(err.norm() / want.norm()))
            assert bool((err <= 4 * u * want.abs() + 8 * u * rms + tiny + extra).all()), (name, float(err.max()), rms)


@pytest.mark.parametrize("B, Sq, Sk, Hq, Hk, D, causal", [(3, 77, 91, 4, 2, 40, False), (1, 1, 300, 2, 1, 128, True), (2, 128, 1025, 2, 2, 128, False), (1, 256, 256, 3, 3, 64, True),
                                                           (1, 2, 4096, 2, 2, 64, False)])
def test_short_half_precision_with_and_without_a_workspace(B, Sq, Sk, Hq, Hk, D, causal, monkeypatch):
    """The powers of two found in each block and those of the kernel before it are the same: the gradients agree bit for bit."""
    from paper_2411_03742_b200 import attention, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(Sq + D)
    q, dout = (torch.randn((B, Sq, Hq, D), generator=g, device="cuda").half() for _ in range(2))
    k, v = (torch.randn((B, Sk, Hk, D), generator=g, device="cuda").half() for _ in range(2))
    dout *= 1e-3
    lens = torch.randint(0, Sk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    out, lse = attention_forward(q, k, v, causal=causal, kv_lens=lens)
    work = torch.full((attention.workspace_bytes(q, k),), 255, dtype=torch.uint8, device="cuda")
    two = attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=lens, workspace=work)
    monkeypatch.setattr(attention, "_one_launch", lambda q, k: True)
    monkeypatch.setattr(attention, "_plans", attention._Plans())
    one = attention_backward(dout, q, k, v, out, lse, causal=causal, kv_lens=lens)
    assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_many_keys_need_a_workspace_in_half_precision():
    import ctypes
    from paper_2411_03742_b200.attention import _Shape, _Tensor
    from paper_2411_03742_b200.binding import EINVAL, load_library
    t = torch.zeros((1, 4097, 1, 64), dtype=torch.float16, device="cuda")
    rows = torch.zeros((1, 1, 8), device="cuda")
    s, x = _Shape(2, 1, 1, 1, 8, 4097, 64, 0, 0.125, None), _Tensor(t.data_ptr(), *t.stride()[:3])
    r = ctypes.byref
    assert load_library().adacons_attn_backward(r(s), r(x), r(x), r(x), r(x), r(x), rows.data_ptr(), r(x), r(x), r(x), None, 0, None) == EINVAL


def test_given_results_that_share_an_input_are_refused():
    from paper_2411_03742_b200 import AdaConsError, attention_backward, attention_forward
    q, k, v, dout = (torch.randn((1, 64, 2, 64), device="cuda").bfloat16() for _ in range(4))
    out, lse = attention_forward(q, k, v)
    for t in (k, v):
        with pytest.raises(AdaConsError):
            attention_forward(q, k, v, out=t)
    for t in (dout, q, k, v, out):
        for name in ("dq", "dk", "dv"):
            with pytest.raises(AdaConsError):
                attention_backward(dout, q, k, v, out, lse, **{name: t})
    one = torch.empty_like(k)
    with pytest.raises(AdaConsError):
        attention_backward(dout, q, k, v, out, lse, dk=one, dv=one)
    want = attention_backward(dout, q, k, v, out, lse)
    packed = torch.empty((1, 64, 6, 64), dtype=torch.bfloat16, device="cuda")      # slices of one buffer are not the same memory
    got = attention_backward(dout, q, k, v, out, lse, dq=packed[:, :, :2], dk=packed[:, :, 2:4], dv=packed[:, :, 4:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
