"""The training operators on a stream other than the current one, with everything they need made by the call."""
import pytest
import torch

pytestmark = pytest.mark.gpu
LATE = 100_000_000          # clock cycles that a stream is kept busy: 50 ms and more


@pytest.mark.parametrize("seq", [100, 700])
def test_a_late_stream_keeps_its_workspace_and_results(seq):
    """The side stream starts long after the call has returned; by then the caller has filled whatever it could allocate."""
    from paper_2411_03742_b200 import Rope, attention_backward, attention_forward
    g = torch.Generator(device="cuda").manual_seed(seq)
    q, k, v, dout = (torch.randn((1, seq, 4, 64), generator=g, device="cuda").bfloat16() for _ in range(4))
    with Rope(64) as rope:
        out, lse = attention_forward(q, k, v, causal=True)
        want = (out, lse, *attention_backward(dout, q, k, v, out, lse, causal=True), rope.apply(q))
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for _ in range(3):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                torch.cuda._sleep(LATE)
            got = (*attention_forward(q, k, v, causal=True, stream=side), *attention_backward(dout, q, k, v, out, lse, causal=True, stream=side),
                   rope.apply(q, stream=side))
            rubbish = [torch.full((n,), float("nan"), device="cuda") for n in (2 * seq * 4, 1024 * 8, 4 * seq * 64 // 2, seq * 4) for _ in range(8)]
            torch.cuda.current_stream().wait_stream(side)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            del got, rubbish
        torch.cuda.synchronize()


def test_results_do_not_take_memory_that_the_current_stream_still_reads():
    """A tensor dropped while work on it is queued goes back to the current stream's memory; a result for another stream must not be made of it."""
    from paper_2411_03742_b200 import Rope, attention_forward
    q = torch.ones((1, 512, 4, 64), device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with Rope(64) as rope:
        for call in (lambda: attention_forward(q, q, q, stream=side), lambda: rope.apply(q, stream=side)):
            torch.cuda.synchronize()
            torch.cuda.empty_cache()
            held = torch.full_like(q, 7.0)
            torch.cuda.synchronize()
            torch.cuda._sleep(LATE)
            copy = held.clone()
            del held
            result = call()
            torch.cuda.synchronize()
            assert (copy == 7.0).all()
            del result


def test_results_freed_early_outlive_the_callers_reading():
    """A result made for the side stream, read on the current one and dropped: the side stream's next call does not get its memory at once."""
    from paper_2411_03742_b200 import Rope
    x = torch.randn((1, 4096, 4, 64), device="cuda")
    side = torch.cuda.Stream()
    with Rope(64) as rope:
        want, other = rope.apply(x), torch.zeros_like(x)
        side.wait_stream(torch.cuda.current_stream())
        y = rope.apply(x, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(LATE)
        copy = y.clone()
        del y
        for _ in range(4):
            rope.apply(other, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(copy, want)


def test_calls_that_are_the_first_of_their_thread():
    """A thread that has made no CUDA call yet, autograd's among them, has no context current until the call makes it so."""
    import threading
    from paper_2411_03742_b200 import AdaCons, Orthogonalizer, Rope, attention_backward, attention_forward
    from paper_2411_03742_b200.attention import attention
    q, dout = (torch.randn((1, 200, 2, 64), device="cuda").bfloat16() for _ in range(2))
    u = torch.randn(300 * 200, device="cuda").bfloat16()
    few, many = torch.randn((8, 4096), device="cuda"), torch.randn((8, 2_000_000), device="cuda")
    out, lse = attention_forward(q, q, q)
    want = attention_backward(dout, q, q, q, out, lse)
    with Rope(64) as rope, Orthogonalizer([(300, 200)], "bf16") as plan, AdaCons(8, 4096) as small, AdaCons(8, 2_000_000) as large:
        made = torch.empty_like(u)
        spare = [torch.empty_like(t) for t in (out, lse, q, q, q, q)]
        rope.apply(q, out=spare[5])
        torch.cuda.synchronize()
        errors = []

        def run(call):
            try:
                call()
            except Exception as e:
                errors.append(repr(e))

        # (a context of another thread must not be rebuilt in between: each call gets a thread of its own)
        for call in (lambda: attention_forward(q, q, q, out=spare[0], lse=spare[1]),
                     lambda: attention_backward(dout, q, q, q, out, lse, dq=spare[2], dk=spare[3], dv=spare[4]),
                     lambda: rope.apply(q, out=spare[5]), lambda: plan.apply(u, made), lambda: small.aggregate(few, few.clone()[0]),
                     lambda: large.aggregate(many, torch.empty_like(many[0]))):
            t = threading.Thread(target=run, args=(call,))
            t.start()
            t.join()
        torch.cuda.synchronize()
        assert not errors, errors
        assert torch.equal(spare[0], out) and torch.equal(spare[1], lse) and all(torch.equal(a, b) for a, b in zip(spare[2:5], want))
        leaves = [q.clone().requires_grad_() for _ in range(3)]
        attention(*leaves).backward(dout)               # the first thing that autograd's thread does on this device, where this test runs alone
        assert all(torch.equal(t.grad, w) for t, w in zip(leaves, want))
