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
