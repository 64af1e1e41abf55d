"""CPU-only checks of what the differentiable forms of the norms, the feed-forward block and the distillation ask of their passes."""
import pytest
import torch


@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("parameters", [False, True])
def test_gate_and_up_are_kept_where_a_gradient_is_recorded(monkeypatch, mode, parameters):
    from paper_2411_03742_b200 import feedforward
    asked = []

    def forward(x, w_gate, w_up, w_down, *, act, keep):
        asked.append(keep)
        hidden = x.new_empty((x.shape[0], w_gate.shape[0]))
        return torch.empty_like(x), hidden if keep else None, hidden.clone() if keep else None

    monkeypatch.setattr(feedforward, "feedforward_forward", forward)
    w = [torch.zeros(s, dtype=torch.bfloat16) for s in ((16, 8), (16, 8), (8, 16))]
    if parameters:
        w = [torch.nn.Parameter(t) for t in w]
    x = torch.zeros((2, 3, 8), dtype=torch.bfloat16)
    with mode():
        y = feedforward.gated_feedforward(x, *w)
    recorded = parameters and mode is torch.enable_grad
    assert asked == [recorded] and y.requires_grad == recorded and y.shape == x.shape


STATUS = r"""
#include <cstdio>
#include "adacons_status.cuh"
static uint32_t word, late;      // `late`: what a kernel of another stream sets between the call's first step and its next
static void between() { word |= late; late = 0; }
cudaError_t cudaMemcpyAsync(void* to, const void* from, size_t, cudaMemcpyKind, cudaStream_t) { *static_cast<uint32_t*>(to) = *static_cast<const uint32_t*>(from); between(); return cudaSuccess; }
cudaError_t cudaMemsetAsync(void* to, int, size_t, cudaStream_t) { *static_cast<uint32_t*>(to) = 0; return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
static void look() { uint32_t v = 9; const int rc = adacons::take_status(&word, &v, nullptr); std::printf("%d %x\n", rc, v); }
int main() {
  look();
  word = 0x100; look(); look();
  late = 0x100; look(); look(); look();
  word = late = 0x100; look(); look();
}
"""


def test_a_status_set_behind_the_look_is_told_by_the_next(tmp_path):
    """The reading of a status word against a runtime of its own, in which another stream's kernel comes between two steps."""
    import os
    import shutil
    import subprocess
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    (tmp_path / "status.cpp").write_text(STATUS)
    home = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(root, "paper_2411_03742_b200", "csrc"), "-I", os.path.join(root, "include"), "-I", os.path.join(home, "include"),
                    "-o", str(tmp_path / "status"), str(tmp_path / "status.cpp")], check=True)
    told = subprocess.run([str(tmp_path / "status")], check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    assert told == ["0 0", "0 100", "0 0", "0 0", "0 100", "0 0", "0 100", "0 0"]


def movable_loads(text):
    """The asm statements without `volatile` that load, whichever of their instructions it is."""
    import re
    found = []
    for start in re.finditer(r"\b(?:asm|__asm__|__asm)\b\s*(\w*)\s*\(", text):
        at, depth = start.end(), 1
        while depth:
            if text[at] == '"':                        # to the end of the literal
                at = re.compile(r'"(?:[^"\\]|\\.)*"').match(text, at).end()
                continue
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        if not start[1].strip("_").startswith("volatile") and re.search(r"\b(ld|ldu|ldmatrix|multimem|atom|red)\b", text[start.start():at]):
            found.append(text[start.start():at])
    return found


def test_loads_stay_behind_their_guards_whatever_comes_before_them():
    """A load in an asm statement without `volatile` may be moved in front of the branch that guards it; it need not be the statement's first instruction."""
    import os
    positive = ['asm("ld.global.nc.u32 %0, [%1];" : "=r"(v) : "l"(p));', 'asm ("{ .reg .pred q; setp.ne.u32 q, %2, 0;" "@q ld.global.u32 %0, [%1]; }" : "=r"(v) : "l"(p), "r"(f(x)));',
                '__asm__("mov.u32 %0, 1; \\"; ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));']
    for text in positive:
        assert movable_loads(f"int a(int);\n{text}\nreturn;") == [text[:-1]], text
        for word in ("volatile", "__volatile__"):
            assert movable_loads(text.replace("(", f" {word}(", 1)) == []
    assert movable_loads('asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));') == []
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_03742_b200", "csrc")
    seen = 0
    for name in sorted(os.listdir(folder)):
        if name.endswith((".cu", ".cuh")):
            text = open(os.path.join(folder, name)).read()
            assert movable_loads(text) == [], name
            seen += text.count("asm")
    assert seen > 50


@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 1e-25, 2.0 ** -61, 2.0 ** 61, 1e30, 3e38])
def test_temperatures_whose_square_or_reciprocal_leave_the_range_are_refused(temperature):
    """tau^2 or 1 / tau would be 0 or infinite in fp32, and the loss 0, infinite or not a number."""
    import ctypes
    from paper_2411_03742_b200 import binding
    from paper_2411_03742_b200.distillation import _Matrix, _Shape, check_distill
    z, ids, top = torch.zeros(4, 50), torch.zeros(4, 5, dtype=torch.int64), torch.zeros(4, 5)
    with pytest.raises(ValueError, match="temperature"):
        check_distill(z, ids, top, temperature, want_cuda=False)
    lib, r = binding.load_library(), ctypes.byref
    # no tokens: nothing is launched
    for tau, code in ((temperature, 1), (2.0 ** -60, 0), (2.0 ** 60, 0)):
        s, m = _Shape(1, 0, 64, 0, 0, 100, 5, tau, 1.0), [_Matrix(None, 128) for _ in range(4)]
        assert lib.adacons_distill_forward(r(s), r(m[0]), r(m[1]), r(m[2]), None, None, None, None) == code
        assert lib.adacons_distill_backward(r(s), None, 1, r(m[0]), r(m[1]), r(m[2]), None, None, r(m[3]), None) == code
        if code == 0:
            check_distill(z, ids, top, tau, want_cuda=False)
