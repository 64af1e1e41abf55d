"""CPU-only checks of the training operators' boundary: the library exports what include/adacons_ops.h
declares, the binding has a prototype for each, bad arguments are refused with a code before any device
is touched, and the rotary angles of every scaling are what their formulas say."""
import ctypes
import math
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN, ELIMIT = 1, 2, 7


@pytest.fixture(scope="module")
def lib():
    from paper_2411_03742_b200 import binding, build
    build.build()
    return binding.load_library()


def declared():
    text = open(os.path.join(ROOT, "include", "adacons_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(adacons_(?:orth|attn|rope)_[a-z_0-9]+)\s*\(", text)))


def test_every_declared_function_is_exported_and_has_a_prototype(lib):
    names = declared()
    assert len(names) == 12, names
    for name in names:
        assert getattr(lib, name).argtypes is not None, name


def test_header_compiles_as_c99(tmp_path):
    import shutil
    import subprocess
    src = tmp_path / "use.c"
    src.write_text('#include "adacons_ops.h"\nint main(void) { adacons_attn_shape s; (void)s; return ADACONS_F16 == 2 ? 0 : 1; }\n')
    cc = shutil.which("gcc") or shutil.which("cc")
    assert cc
    subprocess.run([cc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "use.o")], check=True)


def _orth(lib, dtype=1, d=100, rows=(5,), cols=(7,), offsets=(0,), scaling=0, steps=1, coeffs=(1.0, 0.0, 0.0), eps=0.0, num=None):
    n = len(rows)
    i64 = ctypes.c_int64 * n
    ctx = ctypes.c_void_p()
    return lib.adacons_orth_create(ctypes.byref(ctx), dtype, d, n if num is None else num, i64(*rows), i64(*cols), i64(*offsets), scaling, steps,
                                   (ctypes.c_double * len(coeffs))(*coeffs), eps)


@pytest.mark.parametrize("bad, code", [
    (dict(dtype=2), EINVAL), (dict(d=0), EINVAL), (dict(num=0), EINVAL), (dict(rows=(0,)), EINVAL), (dict(cols=(-1,)), EINVAL),
    (dict(offsets=(-1,)), EINVAL), (dict(offsets=(66,)), EINVAL), (dict(rows=(50,)), EINVAL),
    (dict(rows=(5, 5), cols=(7, 7), offsets=(0, 34)), EINVAL), (dict(scaling=2), EINVAL), (dict(steps=0), EINVAL), (dict(steps=65), EINVAL),
    (dict(coeffs=(1.0, math.nan, 0.0)), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=math.inf), EINVAL),
    (dict(d=1 << 40, rows=((1 << 18) + 1,), cols=(1,)), ELIMIT),
])
def test_orth_refusals(lib, bad, code):
    assert _orth(lib, **bad) == code


def test_orth_null_pointers(lib):
    assert lib.adacons_orth_create(None, 1, 1, 1, None, None, None, 0, 1, None, 0.0) == EINVAL
    assert lib.adacons_orth_apply(None, None, None, None) == EINVAL
    assert lib.adacons_orth_destroy(None) == 0


def _attn(lib, data=1 << 20, strides=(64, 64, 64), **change):
    from paper_2411_03742_b200.attention import _Shape, _Tensor
    fields = dict(dtype=1, batch=2, q_heads=4, kv_heads=2, q_len=3, kv_len=5, head_dim=64, causal=0, scale=0.125, kv_lens=None)
    fields.update(change)
    s, t = _Shape(**fields), _Tensor(data, *strides)
    r = ctypes.byref
    n = ctypes.c_int64()
    return (lib.adacons_attn_forward(r(s), r(t), r(t), r(t), r(t), None, None),
            lib.adacons_attn_backward(r(s), r(t), r(t), r(t), r(t), r(t), None, r(t), r(t), r(t), None, 0, None),
            lib.adacons_attn_workspace_bytes(r(s), r(n)))


@pytest.mark.parametrize("bad, code", [
    (dict(dtype=0), EINVAL), (dict(dtype=3), EINVAL), (dict(batch=-1), EINVAL), (dict(q_heads=0), EINVAL), (dict(q_heads=3), EINVAL), (dict(kv_heads=0), EINVAL),
    (dict(q_len=-1), EINVAL), (dict(kv_len=-1), EINVAL), (dict(head_dim=60), EINVAL), (dict(head_dim=0), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=math.nan), EINVAL), (dict(scale=-1.0), EINVAL), (dict(causal=2), EINVAL), (dict(head_dim=136), ELIMIT), (dict(batch=65536), ELIMIT),
])
def test_attention_refuses_bad_shapes(lib, bad, code):
    assert _attn(lib, **bad) == (code, code, code)


@pytest.mark.parametrize("bad, code", [
    (dict(data=None), EINVAL), (dict(data=(1 << 20) + 8), EALIGN), (dict(strides=(64, 4, 64)), EALIGN), (dict(strides=(0, 64, 64)), EINVAL),
    (dict(strides=(-64, 64, 64)), EINVAL), (dict(), EINVAL),          # the last: no lse, no workspace
])
def test_attention_refuses_bad_tensors(lib, bad, code):
    assert _attn(lib, **bad)[:2] == (code, code)


def test_attention_without_work_succeeds_without_a_device(lib):
    assert _attn(lib, batch=0, data=None) == (0, 0, 0)
    assert _attn(lib, q_len=0, kv_len=0, data=None) == (0, 0, 0)


def test_rope_refusals(lib):
    ctx = ctypes.c_void_p()
    f = (ctypes.c_double * 2)(1.0, 0.5)
    assert lib.adacons_rope_create(None, 4, f, 1.0, 0) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 3, f, 1.0, 0) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 0, f, 1.0, 0) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 4, f, math.inf, 0) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 4, f, 1.0, 2) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 4, (ctypes.c_double * 2)(1.0, math.nan), 1.0, 0) == EINVAL
    assert lib.adacons_rope_create(ctypes.byref(ctx), 8192, f, 1.0, 0) == ELIMIT
    assert lib.adacons_rope_apply(None, None, None, None, None, None, None, 0, 0, None) == EINVAL
    assert lib.adacons_rope_destroy(None) == 0


def test_binding_checks():
    from paper_2411_03742_b200 import attention, orth, rope
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    q, k = z(2, 5, 4, 16), z(2, 7, 2, 16)
    ok = dict(want_cuda=False)
    attention.check_attention(q, k, k, **ok)
    packed = z(2, 5, 8, 16)
    attention.check_attention(packed[:, :, :4], packed[:, :, 4:6], packed[:, :, 6:], **ok)
    for bad in [(q[0], k, k), (q.float(), k, k), (q, k, z(2, 8, 2, 16)), (q, z(2, 7, 3, 16), z(2, 7, 3, 16)), (z(2, 5, 4, 12), z(2, 7, 2, 12), z(2, 7, 2, 12)),
                (z(2, 5, 4, 136), z(2, 7, 2, 136), z(2, 7, 2, 136)), (q, z(1, 7, 2, 16), z(1, 7, 2, 16)), (q, k, k.half()), (z(2, 5, 4, 32)[..., ::2], k, k),
                (z(2, 5, 4, 20)[..., :16], k, k), (z(2, 1, 4, 16).expand(2, 5, 4, 16), k, k)]:
        with pytest.raises(ValueError):
            attention.check_attention(*bad, **ok)
    with pytest.raises(ValueError):
        attention.check_attention(q, k, k, torch.zeros(2, dtype=torch.int64), **ok)
    with pytest.raises(ValueError):
        attention.check_attention(q, k, k, torch.zeros(3, dtype=torch.int32), **ok)
    with pytest.raises(ValueError):
        attention.check_attention(q, k, k, rows=[("lse", torch.zeros(2, 5, 4))], **ok)
    with pytest.raises(ValueError):
        attention.check_attention(q, k, k)                                    # not on a device
    orth.check_vectors(10, "bf16", z(10), z(10), want_cuda=False)
    for bad in [(z(9), z(10)), (z(10), z(10, dt=torch.float32)), (z(20)[::2], z(10)), (z(2, 5), z(10))]:
        with pytest.raises(ValueError):
            orth.check_vectors(10, "bf16", *bad, want_cuda=False)
    x = z(2, 5, 4, 16)
    rope.check_rope(16, x, None, x, want_cuda=False)
    for bad in [(20, x, None, x), (16, x[0], None, x[0]), (16, x.half(), None, x.half()), (16, x, None, z(2, 5, 4, 18)), (16, x, torch.zeros(2, 5), x),
                (16, x, None, z(2, 1, 4, 16).expand(2, 5, 4, 16)), (16, z(2, 5, 4, 32)[..., ::2], None, x)]:
        with pytest.raises(ValueError):
            rope.check_rope(*bad, want_cuda=False)


def test_rotary_frequencies():
    from paper_2411_03742_b200.rope import frequencies
    f, g = frequencies(8, 100.0)
    assert g == 1.0 and f == pytest.approx([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], rel=1e-14)
    lin, g = frequencies(8, 100.0, ("linear", 4.0))
    assert g == 1.0 and lin == pytest.approx([x / 4 for x in f], rel=1e-14)
    ntk, g = frequencies(64, 10000.0, ("ntk", 8.0))
    plain, _ = frequencies(64, 10000.0)
    assert g == 1.0 and ntk[0] == 1.0 and ntk[-1] == pytest.approx(plain[-1] / 8.0, rel=1e-12)   # the definition: the slowest pair, eight times slower
    yarn, g = frequencies(64, 10000.0, ("yarn", 16.0, 4096))
    assert g == pytest.approx(0.1 * math.log(16.0) + 1.0, rel=1e-15)
    turns = [4096 * x / (2 * math.pi) for x in plain]
    for t, x, y in zip(turns, plain, yarn):
        if t > 40:
            assert y == pytest.approx(x, rel=1e-14)
        elif t < 0.8:
            assert y == pytest.approx(x / 16, rel=1e-14)
        else:
            assert x / 16 * (1 - 1e-12) <= y <= x * (1 + 1e-12)
    assert frequencies(8, 100.0, ("linear", 1.0))[0] == f
    for bad in [dict(dim=3), dict(dim=0), dict(dim=8, base=0.0), dict(dim=8, scaling=("linear", 0.5)), dict(dim=8, scaling=("what", 2.0)), dict(dim=2, scaling=("ntk", 2.0))]:
        with pytest.raises(ValueError):
            frequencies(**bad)


def test_aligned_cluster_barriers_meet_as_whole_warps():
    """`barrier.cluster` with `.aligned` is undefined for lanes that arrive apart, and the joins before it let lanes of a ragged tile
    go early: the helper itself brings the warp together, and nothing goes round the helper."""
    csrc = os.path.join(ROOT, "paper_2411_03742_b200", "csrc")
    text = {n: open(os.path.join(csrc, n)).read() for n in ("adacons_tc.cuh", "adacons_attn.cuh", "adacons_orth.cuh", "adacons_rope.cuh")}
    places = [(n, m.start()) for n, t in text.items() for m in re.finditer(r'asm volatile\("barrier\.cluster', t)]
    assert [n for n, _ in places] == ["adacons_tc.cuh"], places
    before = text["adacons_tc.cuh"][:places[0][1]].rstrip().splitlines()
    assert before[-1].strip() == "__syncwarp();"


class _Fake:
    """A tensor as far as the checks look, on a device of any number; its storage is never touched."""

    def __init__(self, shape, dtype=torch.bfloat16, device=1, data=1 << 20):
        self.shape, self.dtype, self.device, self.is_cuda, self.data = torch.Size(shape), dtype, torch.device("cuda", device), True, data

    def stride(self, k=None):
        steps = [math.prod(self.shape[i + 1:]) for i in range(len(self.shape))]
        return tuple(steps) if k is None else steps[k]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def get_device(self):
        return self.device.index

    def data_ptr(self):
        return self.data

    def is_contiguous(self):
        return True


class _FakeLibrary:
    """Notes the device that is current at each call instead of launching anything."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, torch.cuda.current_device(), args))
            return 0
        return call


@pytest.fixture
def fake(monkeypatch):
    """Two devices, 0 current, and a library that launches nothing."""
    from types import SimpleNamespace
    from paper_2411_03742_b200 import attention, orth, rope
    now, library = [0], _FakeLibrary()

    class Device:
        def __init__(self, device):
            self.to = device if isinstance(device, int) else device.index

        def __enter__(self):
            self.was, now[0] = now[0], self.to

        def __exit__(self, *exc):
            now[0] = self.was

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "get_device_properties", lambda device: SimpleNamespace(multi_processor_count=148))
    for module in (attention, orth, rope):
        monkeypatch.setattr(module, "load_library", lambda: library)
        monkeypatch.setattr(module, "_raw_stream", lambda stream, device: 0 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(attention, "_current_device", lambda: now[0])
    monkeypatch.setattr(attention, "_plans", attention._Plans())
    return library


def test_contexts_refuse_tensors_of_another_device(fake):
    from paper_2411_03742_b200 import Orthogonalizer, Rope
    with Orthogonalizer([(4, 8)], "bf16") as plan, Rope(16) as turn:
        assert plan.device == turn.device == 0
        del fake.calls[:]
        for bad in (lambda: plan.apply(_Fake((32,)), _Fake((32,))), lambda: turn.apply(_Fake((1, 2, 3, 16)), out=_Fake((1, 2, 3, 16)))):
            with pytest.raises(ValueError, match="device 1"):
                bad()
        assert not fake.calls
        plan.apply(_Fake((32,), device=0), _Fake((32,), device=0))
        turn.apply(_Fake((1, 2, 3, 16), device=0), out=_Fake((1, 2, 3, 16), device=0))
        assert [c[0] for c in fake.calls] == ["adacons_orth_apply", "adacons_rope_apply"]
        with torch.cuda.device(1):           # the library makes the context's device current by itself
            plan.apply(_Fake((32,), device=0), _Fake((32,), device=0))


def test_attention_runs_on_its_tensors_device(fake):
    from paper_2411_03742_b200 import attention_backward, attention_forward
    q, lse = _Fake((1, 200, 2, 64)), _Fake((1, 2, 200), torch.float32)
    for device in (1, 0):
        q.device = lse.device = torch.device("cuda", device)
        attention_forward(q, q, q, out=q, lse=lse)
        attention_backward(q, q, q, q, q, lse, dq=q, dk=q, dv=q, workspace=_Fake((1 << 20,), torch.uint8, device))
        assert [c[1] for c in fake.calls if c[0] in ("adacons_attn_forward", "adacons_attn_backward")] == [device, device]
        assert torch.cuda.current_device() == 0
        del fake.calls[:]


def test_streams_of_another_device_are_refused(fake):
    from types import SimpleNamespace
    from paper_2411_03742_b200 import Orthogonalizer, Rope, attention_forward
    other = SimpleNamespace(cuda_stream=7, device=torch.device("cuda", 1))
    q, lse = _Fake((1, 200, 2, 64), device=0), _Fake((1, 2, 200), torch.float32, 0)
    with Orthogonalizer([(4, 8)], "bf16") as plan, Rope(16) as turn:
        del fake.calls[:]
        for bad in (lambda: attention_forward(q, q, q, out=q, lse=lse, stream=other), lambda: plan.apply(_Fake((32,), device=0), _Fake((32,), device=0), stream=other),
                    lambda: turn.apply(q, out=q, stream=other)):
            with pytest.raises(ValueError, match="stream"):
                bad()
        assert not fake.calls


def test_what_a_call_on_another_stream_allocates_belongs_to_that_stream(fake, monkeypatch):
    """Made from the current stream's memory, results could meet work still queued there, and a workspace dropped at the
    return what the caller allocates next."""
    from types import SimpleNamespace
    from paper_2411_03742_b200 import Rope, attention, attention_backward, attention_forward, binding, rope
    mine, side = SimpleNamespace(cuda_stream=5, device=torch.device("cuda", 0)), SimpleNamespace(cuda_stream=7, device=torch.device("cuda", 0))
    now, made = [mine], []

    class On:
        def __init__(self, stream):
            self.to = stream

        def __enter__(self):
            self.was, now[0] = now[0], self.to

        def __exit__(self, *exc):
            now[0] = self.was

    class Made(_Fake):
        def __init__(self, shape, dtype):
            super().__init__(shape, dtype, 0)
            self.stream, self.users = now[0], []
            made.append(self)

        def record_stream(self, stream):
            self.users.append(stream)

    monkeypatch.setattr(_Fake, "new_empty", lambda self, shape, dtype=None: Made((shape,) if isinstance(shape, int) else shape, dtype or self.dtype), raising=False)
    monkeypatch.setattr(torch, "empty_like", lambda t, **how: Made(t.shape, t.dtype))
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[0])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device: {5: mine, 7: side}[handle])
    for module in (attention, rope, binding):
        monkeypatch.setattr(module, "_raw_stream", lambda stream, device: (now[0] if stream is None else stream).cuda_stream)
    monkeypatch.setattr(attention, "workspace_bytes", lambda q, k: 4096)
    q, lse = _Fake((1, 400, 2, 64), device=0), _Fake((1, 2, 400), torch.float32, 0)
    with Rope(16) as turn:
        for stream in (side, mine, None):
            del made[:], fake.calls[:]
            results = [*attention_forward(q, q, q, stream=stream), *attention_backward(q, q, q, q, q, lse, stream=stream), turn.apply(q, stream=stream)]
            on = side if stream is side else mine
            assert len(made) == 7 and all(t.stream is on for t in made), "outputs, workspace"
            assert [c[2][-1] for c in fake.calls] == [on.cuda_stream] * 3
            if stream is side:
                assert all(t.users == [mine] for t in results), "freed only after what the caller does with them"
            assert now[0] is mine


def test_a_scale_held_in_a_tensor_is_read_at_every_call(fake):
    from paper_2411_03742_b200 import attention_backward, attention_forward
    q, lse, scale = _Fake((1, 400, 2, 64), device=0), _Fake((1, 2, 400), torch.float32, 0), torch.tensor(0.5)
    work = _Fake((1 << 20,), torch.uint8, 0)
    seen = []
    for factor in (1.0, 4.0, 0.25):
        scale.mul_(factor)
        for call in (lambda: attention_forward(q, q, q, scale=scale, out=q, lse=lse), lambda: attention_backward(q, q, q, q, q, lse, scale=scale, dq=q, dk=q, dv=q, workspace=work)):
            del fake.calls[:]
            call()
            seen.append([c[2][0]._obj.scale for c in fake.calls if c[0] in ("adacons_attn_forward", "adacons_attn_backward")])
    assert seen == [[0.5], [0.5], [2.0], [2.0], [0.5], [0.5]]


def test_a_scale_that_wants_a_gradient_is_refused():
    from paper_2411_03742_b200.attention import attention
    q = torch.zeros((1, 8, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="scale"):
        attention(q, q, q, scale=torch.tensor(0.5, requires_grad=True))


def test_second_derivatives(monkeypatch):
    """Attention says that it has none; the turn, a linear map, has its own back again.  In place of the kernels stand products
    on the CPU that have the formulas' linear structure."""
    from paper_2411_03742_b200 import attention as module
    from paper_2411_03742_b200.rope import _Turn
    monkeypatch.setattr(module, "attention_forward", lambda q, k, v, **how: ((q * k).detach(), torch.zeros(1)))
    monkeypatch.setattr(module, "attention_backward", lambda dout, q, k, v, out, lse, **how: ((dout * k).detach(), (dout * q).detach(), torch.zeros_like(v)))
    x = torch.randn((1, 3, 2, 8), generator=torch.Generator().manual_seed(1), requires_grad=True)
    for f in (lambda x: module.attention(x, x, x).sum(), lambda x: module.attention(x * x, x, x).square().sum()):
        one = torch.autograd.grad(f(x), x, create_graph=True)[0]
        with pytest.raises(NotImplementedError, match="once"):
            torch.autograd.grad(one.square().sum(), x)

    class Turn:                       # (a, b) -> (2 a - b, a + 2 b) and its transpose
        def apply(self, x, positions=None, inverse=False, first=0):
            a, b = x.detach().chunk(2, -1)
            s = -1.0 if inverse else 1.0
            return torch.cat([2 * a - s * b, s * a + 2 * b], -1)

    f = lambda x: _Turn.apply(x * x * x, Turn(), None, 0, False).square().sum()  # noqa: E731
    g = torch.autograd.grad(f(x), x, create_graph=True)[0]
    h = torch.autograd.grad(g.square().sum(), x)[0]
    y = x.detach().double().requires_grad_()              # |R y|^2 = 5 |y|^2
    g2 = torch.autograd.grad(5 * (y ** 3).square().sum(), y, create_graph=True)[0]
    want = torch.autograd.grad(g2.square().sum(), y)[0]
    assert float((h.double() - want).abs().max()) <= 1e-5 * float(want.abs().max())


def test_gradients_that_the_kernel_cannot_read_are_copied(monkeypatch):
    """What autograd hands on may be broadcast, strided or start anywhere: it reaches the kernel aligned, with its values."""
    from paper_2411_03742_b200 import attention as module
    seen = []
    monkeypatch.setattr(module, "attention_forward", lambda q, k, v, **how: (q.detach().clone(), torch.zeros(1)))
    monkeypatch.setattr(module, "attention_backward", lambda dout, q, k, v, out, lse, **how: (seen.append(dout), (dout, k, v))[1])
    x = torch.randn((2, 3, 2, 16), generator=torch.Generator().manual_seed(1)).bfloat16().requires_grad_()
    weight = torch.randn(200, generator=torch.Generator().manual_seed(2)).bfloat16()
    for use, want in ((lambda y: (torch.cat([torch.zeros(3, dtype=y.dtype), y.flatten()]) * weight[:195]).sum(), weight[3:195].view(x.shape)),
                      (lambda y: y.sum(), torch.ones_like(x)), (lambda y: (torch.cat([y, y[..., :4]], -1).flatten(2) * weight[:40]).sum(), None)):
        x.grad = None
        use(module.attention(x, x.detach(), x.detach())).backward()
        dout = seen.pop()
        assert dout.data_ptr() % 16 == 0 and dout.stride(3) == 1 and all(s % 8 == 0 and s > 0 for s in dout.stride()[:3])
        if want is not None:
            assert torch.equal(dout, want)


def test_turns_of_nothing_in_any_layout():
    """Tensors without elements share the address 0 whatever their strides: that does not make them an in-place call."""
    from paper_2411_03742_b200 import rope
    for shape in ((2, 0, 6, 16), (0, 3, 6, 16)):
        x = torch.zeros(shape)[:, :, :4]
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        assert x.data_ptr() == out.data_ptr() == 0
        rope.check_rope(16, x, None, out, want_cuda=False)
    x = torch.zeros((2, 3, 6, 16))
    with pytest.raises(ValueError, match="in place"):
        rope.check_rope(16, x[:, :, :4], None, torch.as_strided(x, (2, 3, 4, 16), (192, 64, 16, 1)), want_cuda=False)


def test_what_the_readme_imports_can_be_called():
    """Every name that the README's snippets import from the package is a class or a function, not a module of that name."""
    import importlib
    text = open(os.path.join(ROOT, "README.md")).read()
    found = re.findall(r"^from (paper_2411_03742_b200[\w.]*) import ([\w, ]+)$", text, flags=re.M)
    names = [(module, name.strip()) for module, several in found for name in several.split(",")]
    assert {"AdaCons", "Orthogonalizer", "Rope", "attention", "attention_forward", "attention_backward"} <= {n for _, n in names}
    for module, name in names:
        assert callable(getattr(importlib.import_module(module), name)), (module, name)


def test_results_in_the_place_of_what_is_read_are_refused(lib):
    """Written where other blocks still read, they would be right or wrong by chance.  Checked before any device is touched."""
    from paper_2411_03742_b200.attention import _Shape, _Tensor
    s = _Shape(1, 2, 4, 2, 3, 5, 64, 0, 0.125, None)
    at = lambda n: _Tensor((1 << 20) + (n << 16), 1024, 256, 64)  # noqa: E731
    r, rows = ctypes.byref, 1 << 30
    q, k, v, out, dout, dq, dk, dv = (at(n) for n in range(8))
    assert lib.adacons_attn_forward(r(s), r(q), r(k), r(v), r(k), rows, None) == EINVAL
    assert lib.adacons_attn_forward(r(s), r(q), r(k), r(v), r(v), rows, None) == EINVAL
    back = lambda *g: lib.adacons_attn_backward(r(s), r(dout), r(q), r(k), r(v), r(out), rows, *(r(t) for t in g), 1 << 29, 1 << 20, None)  # noqa: E731
    for t in (dout, q, k, v, out):
        assert back(t, dk, dv) == back(dq, t, dv) == back(dq, dk, t) == EINVAL
    assert back(dq, dk, dk) == back(dq, dq, dv) == EINVAL
