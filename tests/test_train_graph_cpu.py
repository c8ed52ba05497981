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


@pytest.mark.parametrize("needs", [(True, False, False), (False, True, False), (True, True, False), (False, False, True),
                                   (True, True, True)], ids=str)
def test_collect_keeps_expert_rows_for_the_gates_alone(monkeypatch, needs):
    """T * k rows that no gradient reads are not held: a frozen router's gates need none of them."""
    monkeypatch.setattr(train, "_collect", lambda y, *_: y[:2] * 1.0)
    calls = []

    def collect_backward(d_out, y, positions, tokens, gates, span, y_type):
        calls.append((y is not None, y_type))
        return (None if y_type is None else torch.ones(4, 8, dtype=y_type)), (None if y is None else torch.ones(2, 2))

    monkeypatch.setattr(train, "_collect_backward", collect_backward)
    y, gates, residual = (torch.ones(s).requires_grad_(n) for s, n in zip(((4, 8), (2, 2), (2, 8)), needs))
    places = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    out = train._graph()["collect"](y, gates, residual, *places, None, None)
    held = [t for t in out.grad_fn.saved_tensors if t is not None]
    assert any(t.data_ptr() == y.data_ptr() for t in held) == needs[1]
    assert any(t.data_ptr() == gates.data_ptr() for t in held) == (needs[0] or needs[1])
    out.backward(torch.ones(2, 8))
    assert calls == ([(needs[1], torch.float32 if needs[0] else None)] if needs[0] or needs[1] else [])
    assert [t.grad is not None for t in (y, gates, residual)] == list(needs)
