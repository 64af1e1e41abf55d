"""CPU-only checks of the norms', the feed-forward block's and the distillation's boundary: what the header declares is exported, bad arguments are
refused before any device is touched, and the calls run on the device and stream of their tensors."""
import ctypes
import math
import os
import re

import pytest
import torch

from test_ops_host import EALIGN, EINVAL, ELIMIT, ROOT, _Fake, _FakeLibrary, lib  # noqa: F401

NAMES = {"adacons_norm_forward", "adacons_norm_backward", "adacons_norm_workspace_bytes", "adacons_ffn_forward", "adacons_ffn_backward", "adacons_ffn_workspace_bytes",
         "adacons_ffn_get_status", "adacons_distill_forward", "adacons_distill_backward", "adacons_selftest_ffn"}
r = ctypes.byref
AT = 1 << 20


def test_every_declared_function_is_exported_and_has_a_prototype(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "adacons_ops.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(adacons_(?:(?:norm|ffn|distill)_[a-z_0-9]+|selftest_ffn))\s*\(", text))
    assert declared == NAMES
    for name in NAMES:
        assert getattr(lib, name).argtypes is not None, name
        args = re.search(rf"\b{name}\s*\((.*?)\)\s*;", text, flags=re.S)[1]
        assert len(getattr(lib, name).argtypes) == args.count(",") + 1, name


def test_loads_stay_behind_their_guards():
    """A load in an asm statement without `volatile` may be moved in front of the branch that guards it, to an address that does not exist."""
    folder = os.path.join(ROOT, "paper_2411_03742_b200", "csrc")
    for name in sorted(os.listdir(folder)):
        if name.endswith((".cu", ".cuh")):
            for asm in re.findall(r"\basm\s*\(([^;]*);", open(os.path.join(folder, name)).read()):
                assert not re.search(r"\b(ld|ldmatrix|multimem)\b", asm), (name, asm[:80])


# ---- norms ----------------------------------------------------------------------------------------------
def _norm(lib, data=AT, apart=1 << 16, pre=AT + (1 << 19), post=AT + (1 << 18), rows=1 << 30, **change):
    from paper_2411_03742_b200.norms import _Rows, _Shape
    fields = dict(stream_dtype=1, dtype=1, batch=2, len=3, dim=64, gate=2, gate_by=1, gate_dtype=0, post_dtype=0, pre_dtype=1, scale=1.0, eps=1e-6)
    fields.update(change)
    s = _Shape(**fields)
    t = [_Rows(data and data + i * apart, 192, 64) for i in range(8)]
    forward = lib.adacons_norm_forward(r(s), r(t[0]), r(t[1]), r(t[2]), post, pre, r(t[3]), r(t[4]), rows, None)
    back = lib.adacons_norm_backward(r(s), r(t[0]), r(t[1]), r(t[2]), r(t[3]), r(t[4]), post, pre, rows, r(t[5]), r(t[6]), r(t[7]), 1 << 31, 1 << 32, None, 0, None)
    return forward, back


@pytest.mark.parametrize("bad, code", [
    (dict(dtype=3), EINVAL), (dict(stream_dtype=2), EINVAL), (dict(batch=-1), EINVAL), (dict(len=-1), EINVAL), (dict(dim=0), EINVAL), (dict(gate=4), EINVAL), (dict(gate=-1), EINVAL),
    (dict(gate_by=3), EINVAL), (dict(gate_dtype=2), EINVAL), (dict(post_dtype=3), EINVAL), (dict(pre_dtype=2), EINVAL), (dict(scale=math.nan), EINVAL), (dict(scale=math.inf), EINVAL),
    (dict(eps=0.0), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=math.inf), EINVAL), (dict(dim=16385), ELIMIT), (dict(batch=1 << 16, len=1 << 16), ELIMIT),
    (dict(data=None), EINVAL), (dict(data=AT + 1), EALIGN), (dict(pre=AT + 1), EALIGN), (dict(post=AT + 2), EALIGN), (dict(apart=0), EINVAL)])
def test_norm_refusals(lib, bad, code):
    assert _norm(lib, **bad)[0] == code
    assert _norm(lib, **bad)[1] == code or bad == dict(data=None)         # back: nothing but x' has a gradient then


def test_norm_null_pointers_and_nothing_to_do(lib):
    assert lib.adacons_norm_forward(*[None] * 10) == EINVAL and lib.adacons_norm_backward(*[None] * 15, 0, None) == EINVAL
    n = ctypes.c_int64()
    assert lib.adacons_norm_workspace_bytes(None, r(n)) == EINVAL
    assert _norm(lib, rows=None)[0] == EINVAL
    assert _norm(lib, batch=0, data=None, rows=None)[0] == 0 and _norm(lib, len=0, data=None, rows=None)[0] == 0


def test_norm_checks():
    from paper_2411_03742_b200.norms import check_norm
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, w = z(2, 5, 48), z(48, dt=torch.float32)
    ok = dict(want_cuda=False)
    check_norm(x, x, z(2, 48), w, w, "tanh", **ok)
    check_norm(x.float(), x, z(48), z(48), w, **ok)
    check_norm(x.float(), None, pre=w, dtype=torch.float16, **ok)
    check_norm(x[0], x[0], z(5, 48), **ok)
    check_norm(z(2, 5, 50)[..., :48], z(5, 2, 48).transpose(0, 1), **ok)
    f32 = torch.float32
    for args, how in [((x[0, 0], x[0, 0]), {}), ((z(2, 5, 0), z(2, 5, 0)), {}), ((z(1, 1, 16385), z(1, 1, 16385)), {}), ((x.double(), x.double()), {}), ((x, x.half()), {}),
                      ((x, x.float()), {}), ((x, z(2, 5, 47)), {}), ((x, z(2, 5, 96)[..., ::2]), {}), ((x, None), {}), ((x, None, z(48)), dict(pre=w)), ((x, None, None, w), dict(pre=w)),
                      ((x, x, z(47)), {}), ((x, x, z(3, 48)), {}), ((x, x, z(2, 4, 48)), {}), ((x[0], x[0], z(2, 5, 48)), {}), ((x, x, z(48).half()), {}), ((x, x, None, z(47)), {}),
                      ((x, x, None, None, z(48).half()), {}), ((x, x), dict(gate_by="sigmoid")), ((x, x, z(48)), dict(gate_by="relu")), ((x, x), dict(scale=math.nan)),
                      ((x, x), dict(eps=0.0)), ((x, x), dict(dtype=f32)), ((x, x), dict(like_x=[("out", z(2, 5, 48).half())])), ((x, x), dict(like_x=[("out", z(2, 1, 48).expand(2, 5, 48))])),
                      ((x, x), dict(rows=z(2, 5, dt=f32))), ((x, x), dict(rows=z(2, 2, 5))), ((x, x, z(48)), dict(like_gate=[("dgate", z(48, dt=f32))])),
                      ((x, x, None, w), dict(like_post=[("dpost", z(48))]))]:
        with pytest.raises(ValueError):
            check_norm(*args, **how, **ok)
    with pytest.raises(ValueError, match="CUDA"):
        check_norm(x, x)


# ---- feed-forward ---------------------------------------------------------------------------------------
def _ffn(lib, data=AT, apart=1 << 16, stride=128, work=1 << 30, size=1 << 40, **change):
    from paper_2411_03742_b200.feedforward import _Matrix, _Shape
    fields = dict(dtype=1, tokens=5, dim=64, hidden=128, act=0)
    fields.update(change)
    s = _Shape(**fields)
    m = [_Matrix(data and data + i * apart, stride) for i in range(11)]
    n = ctypes.c_int64()
    return (lib.adacons_ffn_forward(r(s), *(r(x) for x in m[:7]), work, size, None), lib.adacons_ffn_backward(r(s), *(r(x) for x in m), work, size, None),
            lib.adacons_ffn_workspace_bytes(r(s), 1, r(n)))


@pytest.mark.parametrize("bad, code", [(dict(dtype=0), EINVAL), (dict(dtype=3), EINVAL), (dict(tokens=-1), EINVAL), (dict(dim=60), EINVAL), (dict(dim=0), EINVAL), (dict(hidden=4), EINVAL),
                                       (dict(act=4), EINVAL), (dict(act=-1), EINVAL), (dict(tokens=(1 << 24) + 1), ELIMIT), (dict(dim=(1 << 18) + 8), ELIMIT), (dict(hidden=(1 << 18) + 8), ELIMIT)])
def test_ffn_refuses_bad_shapes(lib, bad, code):
    assert _ffn(lib, **bad) == (code, code, code)


@pytest.mark.parametrize("bad, code", [(dict(data=None), EINVAL), (dict(data=AT + 8), EALIGN), (dict(stride=132), EALIGN), (dict(stride=56), EINVAL), (dict(stride=-128), EINVAL),
                                       (dict(apart=0), EINVAL), (dict(work=None), EINVAL), (dict(work=AT + 8), EALIGN), (dict(size=100), EINVAL)])
def test_ffn_refuses_bad_matrices(lib, bad, code):
    assert _ffn(lib, **bad)[:2] == (code, code)


def test_ffn_workspace_and_nothing_to_do(lib):
    from paper_2411_03742_b200.feedforward import _Shape
    n = ctypes.c_int64()
    for tokens, hidden, dtype in ((5, 128, 1), (1 << 24, 1 << 18, 2)):
        s = _Shape(dtype, tokens, 64, hidden, 0)
        one = -(-tokens * hidden * 2 // 256) * 256
        assert lib.adacons_ffn_workspace_bytes(r(s), 0, r(n)) == 0 and n.value == one
        assert lib.adacons_ffn_workspace_bytes(r(s), 1, r(n)) == 0 and n.value == 3 * one + (512 if dtype == 2 else 0)
    assert _ffn(lib, tokens=0, data=AT, work=None)[0] == 0
    assert lib.adacons_ffn_forward(*[None] * 9, 0, None) == EINVAL and lib.adacons_ffn_backward(*[None] * 13, 0, None) == EINVAL


def test_ffn_checks():
    from paper_2411_03742_b200.feedforward import check_feedforward
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, w, d = z(5, 64), z(128, 64), z(64, 128)
    ok = dict(want_cuda=False)
    check_feedforward(x, w, w, d, "gelu", like_hidden=[("gate", z(5, 128))], **ok)
    check_feedforward(z(5, 80)[:, :64], w, w, d, **ok)
    for args, how in [((x[None], w, w, d), {}), ((x.float(), w, w, d), {}), ((x, w.half(), w, d), {}), ((x, w, z(120, 64), d), {}), ((x, w, w, w), {}), ((x, w, w, d, "swish"), {}),
                      ((z(5, 60), z(128, 60), z(128, 60), z(60, 128)), {}), ((z(5, 68)[:, :64], w, w, d), {}), ((z(64, 5).T, w, w, d), {}), ((z(1, 64).expand(5, 64), w, w, d), {}),
                      ((x, w, w, d), dict(like_x=[("out", z(5, 72))])), ((x, w, w, d), dict(like_hidden=[("gate", z(5, 128).half())])), ((x, w, w, d), dict(like_down=[("dw_down", w)]))]:
        with pytest.raises(ValueError):
            check_feedforward(*args, **how, **ok)
    with pytest.raises(ValueError, match="CUDA"):
        check_feedforward(x, w, w, d)


# ---- distillation ---------------------------------------------------------------------------------------
def _distill(lib, data=AT, apart=1 << 16, labels=AT + (1 << 19), loss=1 << 30, rows=1 << 31, **change):
    from paper_2411_03742_b200.distillation import _Matrix, _Shape
    fields = dict(dtype=1, teacher_dtype=0, ids_bits=64, labels_bits=64, tokens=3, vocab=100, top=5, temperature=2.0, mix=0.5)
    fields.update(change)
    s = _Shape(**fields)
    m = [_Matrix(data and data + i * apart, 128) for i in range(4)]
    return (lib.adacons_distill_forward(r(s), r(m[0]), r(m[1]), r(m[2]), labels, loss, rows, None),
            lib.adacons_distill_backward(r(s), loss, 1, r(m[0]), r(m[1]), r(m[2]), labels, rows, r(m[3]), None))


@pytest.mark.parametrize("bad, code", [
    (dict(dtype=3), EINVAL), (dict(teacher_dtype=-1), EINVAL), (dict(ids_bits=16), EINVAL), (dict(labels_bits=8), EINVAL), (dict(tokens=-1), EINVAL), (dict(vocab=0), EINVAL),
    (dict(top=0), EINVAL), (dict(top=1025), ELIMIT), (dict(vocab=(1 << 30) + 1), ELIMIT), (dict(tokens=(1 << 27) + 1), ELIMIT), (dict(temperature=0.0), EINVAL),
    (dict(temperature=math.inf), EINVAL), (dict(temperature=math.nan), EINVAL), (dict(mix=-0.1), EINVAL), (dict(mix=1.1), EINVAL), (dict(mix=math.nan), EINVAL), (dict(data=None), EINVAL),
    (dict(data=AT + 1), EALIGN), (dict(labels=None), EINVAL), (dict(labels=AT + 4), EALIGN), (dict(loss=None), EINVAL), (dict(rows=None), EINVAL), (dict(loss=AT), EINVAL)])
def test_distill_refusals(lib, bad, code):
    got = _distill(lib, **bad)
    assert got[0] == code and (got[1] == code or "loss" in bad)


def test_distill_null_pointers_and_nothing_to_do(lib):
    assert lib.adacons_distill_forward(*[None] * 8) == EINVAL and lib.adacons_distill_backward(None, None, 0, *[None] * 7) == EINVAL
    assert _distill(lib, tokens=0, data=None, labels=None, loss=None, rows=None) == (0, 0)


def test_distill_checks():
    from paper_2411_03742_b200.distillation import check_distill, distill, distill_forward
    z, ids, top, y = torch.zeros(4, 50), torch.zeros(4, 5, dtype=torch.int64), torch.zeros(4, 5), torch.zeros(4, dtype=torch.int64)
    ok = dict(want_cuda=False)
    check_distill(z, ids, top, 2.0, y, 0.5, **ok)
    check_distill(torch.zeros(4, 60)[:, :50].half(), ids.int(), top.bfloat16(), 1.0, y.int(), 0.0, **ok)
    for args, how in [((z[0], ids, top, 1.0), {}), ((z.double(), ids, top, 1.0), {}), ((z, ids.short(), top, 1.0), {}), ((z, ids, top.long(), 1.0), {}), ((z, ids, top[:, :4], 1.0), {}),
                      ((z, ids[:3], top[:3], 1.0), {}), ((z, torch.zeros(4, 1025, dtype=torch.int64), torch.zeros(4, 1025), 1.0), {}), ((z, ids[:, :0], top[:, :0], 1.0), {}),
                      ((z, ids, top, 0.0), {}), ((z, ids, top, math.nan), {}), ((z, ids, top, 1.0, y, 1.5), {}), ((z, ids, top, 1.0, y[:3], 0.5), {}), ((z, ids, top, 1.0, y.float(), 0.5), {}),
                      ((torch.zeros(4, 100)[:, ::2], ids, top, 1.0), {}), ((z, ids, top, 1.0), dict(loss=torch.zeros(3))), ((z, ids, top, 1.0), dict(rows=torch.zeros(4, 2))),
                      ((z, ids, top, 1.0), dict(out=z.half())), ((z, ids, top, 1.0), dict(out=torch.zeros(1, 50).expand(4, 50))), ((z, ids, top, 1.0), dict(dloss=torch.zeros(4).double()))]:
        with pytest.raises(ValueError):
            check_distill(*args, **how, **ok)
    with pytest.raises(ValueError, match="CUDA"):
        check_distill(z, ids, top, 1.0)
    with pytest.raises(ValueError, match="mix"):
        distill_forward(z, ids, top, labels=y)
    for how in (dict(temperature=torch.tensor(2.0, requires_grad=True)), dict(labels=y, mix=torch.tensor(0.5, requires_grad=True))):
        with pytest.raises(ValueError, match="gradient"):
            distill(z, ids, top, **how)
    with pytest.raises(ValueError, match="gradient"):
        distill(z, ids, top.clone().requires_grad_())


# ---- devices and streams --------------------------------------------------------------------------------
@pytest.fixture
def fake(monkeypatch):
    """Two devices, 0 current, and a library that launches nothing."""
    from paper_2411_03742_b200 import calls, distillation, feedforward, norms
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
    monkeypatch.setattr(calls, "_current_device", lambda: now[0])
    for module in (norms, feedforward, distillation):
        monkeypatch.setattr(module, "load_library", lambda: library)
        for plans in ("_plans", "_back_plans"):
            monkeypatch.setattr(module, plans, calls.Plans())
    for module in (calls, norms, feedforward, distillation):
        monkeypatch.setattr(module, "_raw_stream", lambda stream, device: 0 if stream is None else stream.cuda_stream)
    return library


def _calls(device, stream=None):
    """Every pass once on tensors of a device, with everything it writes given."""
    from paper_2411_03742_b200 import (distill_backward, distill_forward, feedforward_backward, feedforward_forward, residual_norm_backward, residual_norm_forward)
    count = [0]

    def t(*shape, dtype=torch.bfloat16):
        count[0] += 1
        return _Fake(shape, dtype, device, (1 << 20) + (count[0] << 24))

    f32, i64 = torch.float32, torch.int64
    x, w = t(2, 3, 64), t(64, dtype=f32)
    rows = t(2, 2, 3, dtype=f32)
    yield lambda: residual_norm_forward(x, t(2, 3, 64), pre=w, out=t(2, 3, 64), normed=t(2, 3, 64), rows=rows, stream=stream)
    yield lambda: residual_norm_backward(t(2, 3, 64), t(2, 3, 64), x, t(2, 3, 64), rows, pre=w, dx=t(2, 3, 64), df=t(2, 3, 64), dpre=t(64, dtype=f32),
                                         workspace=t(1 << 20, dtype=torch.uint8), stream=stream)
    m = [t(5, 64), t(128, 64), t(128, 64), t(64, 128)]
    yield lambda: feedforward_forward(*m, out=t(5, 64), gate=t(5, 128), up=t(5, 128), workspace=t(1 << 20, dtype=torch.uint8), stream=stream)
    yield lambda: feedforward_backward(t(5, 64), *m, t(5, 128), t(5, 128), dx=t(5, 64), dw_gate=t(128, 64), dw_up=t(128, 64), dw_down=t(64, 128),
                                       workspace=t(1 << 20, dtype=torch.uint8), stream=stream)
    z, ids, top = t(4, 50), t(4, 5, dtype=i64), t(4, 5, dtype=f32)
    yield lambda: distill_forward(z, ids, top, loss=t(4, dtype=f32), rows=t(2, 4, dtype=f32), stream=stream)
    yield lambda: distill_backward(t(4, dtype=f32), z, ids, top, t(2, 4, dtype=f32), out=t(4, 50), stream=stream)


PASSES = ["adacons_norm_forward", "adacons_norm_backward", "adacons_ffn_forward", "adacons_ffn_backward", "adacons_distill_forward", "adacons_distill_backward"]


def test_calls_run_on_their_tensors_device(fake):
    for device in (1, 0, 1):
        del fake.calls[:]
        for call in _calls(device):
            call()
        made = [(name, at) for name, at, _ in fake.calls if name in PASSES]
        assert made == [(name, device) for name in PASSES]
        assert torch.cuda.current_device() == 0


def test_streams_of_another_device_are_refused(fake):
    from types import SimpleNamespace
    other = SimpleNamespace(cuda_stream=7, device=torch.device("cuda", 1))
    for call in _calls(0, other):
        with pytest.raises(ValueError, match="stream"):
            call()
    assert not [c for c in fake.calls if c[0] in PASSES]


def test_results_in_the_place_of_what_is_read_are_refused(fake):
    """Written where other blocks still read, or one over another, they would be right or wrong by chance."""
    from paper_2411_03742_b200 import (distill_backward, distill_forward, feedforward_backward, feedforward_forward, residual_norm_backward, residual_norm_forward)
    at = iter(range(1 << 24, 1 << 40, 1 << 24))
    t = lambda *s, dtype=torch.bfloat16: _Fake(s, dtype, 0, next(at))  # noqa: E731
    f32, i64 = torch.float32, torch.int64
    x, f, w, rows = t(2, 3, 64), t(2, 3, 64), t(64, dtype=f32), t(2, 2, 3, dtype=f32)
    work = t(1 << 20, dtype=torch.uint8)
    fine = dict(out=t(2, 3, 64), normed=t(2, 3, 64), rows=rows)
    residual_norm_forward(x, f, pre=w, **fine)
    residual_norm_forward(x, f, pre=w, **{**fine, "out": x})
    for bad in (dict(out=f), dict(normed=x), dict(normed=f), dict(normed=fine["out"])):
        with pytest.raises(ValueError):
            residual_norm_forward(x, f, pre=w, **{**fine, **bad})
    d, dn = t(2, 3, 64), t(2, 3, 64)
    fine = dict(dx=t(2, 3, 64), df=t(2, 3, 64), dpre=t(64, dtype=f32), workspace=work)
    residual_norm_backward(d, dn, x, f, rows, pre=w, **fine)
    residual_norm_backward(d, dn, x, f, rows, pre=w, **{**fine, "dx": d})
    for bad in (dict(dx=x), dict(dx=f), dict(dx=dn), dict(df=d), dict(df=f), dict(df=fine["dx"]), dict(dpre=w)):
        with pytest.raises(ValueError):
            residual_norm_backward(d, dn, x, f, rows, pre=w, **{**fine, **bad})
    m = [t(5, 64), t(128, 64), t(128, 64), t(64, 128)]
    fine = dict(out=t(5, 64), gate=t(5, 128), up=t(5, 128), workspace=work)
    feedforward_forward(*m, **fine)
    for bad in (dict(out=m[0]), dict(gate=fine["up"])):
        with pytest.raises(ValueError):
            feedforward_forward(*m, **{**fine, **bad})
    dy, g, u = t(5, 64), t(5, 128), t(5, 128)
    fine = dict(dx=t(5, 64), dw_gate=t(128, 64), dw_up=t(128, 64), dw_down=t(64, 128), workspace=work)
    feedforward_backward(dy, *m, g, u, **fine)
    for bad in (dict(dx=dy), dict(dx=m[0]), dict(dw_gate=m[1]), dict(dw_up=fine["dw_gate"]), dict(dw_down=m[3])):
        with pytest.raises(ValueError):
            feedforward_backward(dy, *m, g, u, **{**fine, **bad})
    z, ids, top = t(4, 50), t(4, 5, dtype=i64), t(4, 5, dtype=f32)
    loss, rows = t(4, dtype=f32), t(2, 4, dtype=f32)
    distill_forward(z, ids, top, loss=loss, rows=rows)
    same = _Fake((4,), f32, 0, rows.data)
    with pytest.raises(ValueError):
        distill_forward(z, ids, top, loss=same, rows=rows)
    distill_backward(loss, z, ids, top, rows, out=z)
    wide = _Fake((4, 50), torch.bfloat16, 0, ids.data)
    with pytest.raises(ValueError):
        distill_backward(loss, z, ids, top, rows, out=wide)


def test_what_a_call_keeps_is_its_layout(fake):
    """A scale, a temperature or a mix held in a tensor is read at every call."""
    from paper_2411_03742_b200 import distill_forward, residual_norm_forward
    t = lambda *s, dtype=torch.bfloat16, at=[1 << 20]: _Fake(s, dtype, 0, at.__setitem__(0, at[0] + (1 << 20)) or at[0])  # noqa: E731
    value, seen = torch.tensor(0.5), []
    x, f, out, rows = t(2, 3, 64), t(2, 3, 64), t(2, 3, 64), t(2, 2, 3, dtype=torch.float32)
    z, ids, top, loss, L = t(4, 50), t(4, 5, dtype=torch.int64), t(4, 5), t(4, dtype=torch.float32), t(2, 4, dtype=torch.float32)
    for factor in (1.0, 3.0, 1.0 / 3):
        value.mul_(factor)
        del fake.calls[:]
        residual_norm_forward(x, f, scale=value, out=out, rows=rows)
        distill_forward(z, ids, top, temperature=value, loss=loss, rows=L)
        seen.append((fake.calls[0][2][0]._obj.scale, fake.calls[1][2][0]._obj.temperature))
    assert seen == [(0.5, 0.5), (1.5, 1.5), (0.5, 0.5)]


def test_waits_of_the_feedforward_kernels_are_bounded():
    """Every wait of the sources is the bounded one, and no cluster barrier is reached by a part of a warp."""
    csrc = os.path.join(ROOT, "paper_2411_03742_b200", "csrc")
    for name in ("adacons_ffn.cuh", "adacons_norm.cuh", "adacons_distill.cuh"):
        text = open(os.path.join(csrc, name)).read()
        assert not re.search(r"mbar_try_wait\(|mbarrier\.(try_)?wait|while \(true\)|for \(;;\)|barrier\.cluster|multicast", text), name
