"""What the trainer's operators keep and make in torch's graphs, without a GPU:
their kernels' calls are replaced by plain ones."""

import pytest
import torch

from paper_2609_25442_amd import train


@pytest.fixture
def received(monkeypatch):
    """The gradients that the activation's backward is handed."""
    seen = []

    def activate(x, activation, gated, checkpoint, out_dtype):
        if not checkpoint:
            return x * 2, None, None
        return x * 2, torch.zeros(x.shape, dtype=torch.float8_e4m3fn), torch.ones(x.shape[0], 1)

    monkeypatch.setattr(train, "_activate", activate)
    monkeypatch.setattr(train, "_activate_backward", lambda d, saved, scales, *more: d * 2)
    apply = train._graph()["activate"]
    function = apply.__self__
    plain = function.backward

    def watch(ctx, *grads):
        seen.append(grads)
        return plain(ctx, *grads)

    monkeypatch.setattr(function, "backward", staticmethod(watch))
    return apply, seen


@pytest.mark.parametrize("checkpoint", [True, False])
def test_no_gradients_are_made_for_a_checkpoint(received, checkpoint):
    """Zeros of the codes' and scales' shapes would be as large as the checkpoint itself."""
    apply, seen = received
    x = torch.ones(4, 256, requires_grad=True)
    out = apply(x, "silu", False, checkpoint, None)[0]
    out.backward(torch.ones_like(out))
    assert [g is None for g in seen[0]] == [False, True, True]
    assert torch.all(x.grad == 2)


def test_an_activation_whose_result_got_no_gradient_has_none(received):
    apply, seen = received

    class Nothing(torch.autograd.Function):
        @staticmethod
        def forward(ctx, t):
            return t.clone()

        @staticmethod
        def backward(ctx, d):
            return None

    x, y = (torch.ones(2, 128, requires_grad=True) for _ in range(2))
    (Nothing.apply(apply(x, "silu", False, True, None)[0]) + y).sum().backward()
    assert x.grad is None or not x.grad.any()
    assert torch.all(y.grad == 1)
