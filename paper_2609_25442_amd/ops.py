"""Operators on a rank's tensors: what an MoE layer computes with the weights
that unpacking leaves on a rollout rank (norm, router, products with plain and
stacked weights, the sum of a token's expert rows), and the router's gradient
for the trainer.

Each function makes its outputs with torch, enqueues one to three HIP kernels of
libwb on the stream (the current one by default) and returns. Tensors are
float32, bfloat16 or float8_e4m3fn in the memory of the current device; rows
may lie any distance apart. fp8 activations go with float32 scales of one row
and 128 columns, [rows, ceil(cols / 128)]; fp8 weights with those of 128x128
blocks, as unpacking writes them. Arguments that do not fit raise WbError.
Only ``route`` has a gradient: the others serve a rollout rank's tensors, and
raise WbError for one that requires a gradient while gradients are recorded (a
differentiable ``route``'s gates go into ``combine`` detached). Tensors with
a forward-mode tangent are refused by all.
"""

from __future__ import annotations

import collections
import ctypes

from . import DTYPES, WB_EINVAL, WB_EUNSUPPORTED, WbError, _args, lib

ACTIVATIONS = {"none": 0, "silu": 1, "gelu": 2}
_torch = None
_fn = {}


def _address(name: str) -> int:
    """Address of a C entry, for the extension to call."""
    p = _fn.get(name)
    if p is None:
        p = _fn[name] = ctypes.cast(getattr(lib, name), ctypes.c_void_p).value
    return p


def _refused(r):
    if isinstance(r, str):
        raise WbError(WB_EINVAL, r)
    raise WbError(r, lib.wb_last_error().decode())


def _here():
    """(current device, handle of its current stream)."""
    global _torch
    if _torch is None:
        import torch

        _torch = torch
    d = _torch.cuda.current_device()
    return d, _torch._C._cuda_getCurrentRawStream(d)


def _type(name, choices, what):
    if name is None:
        return -1
    try:
        return choices[name]
    except (KeyError, TypeError):
        raise WbError(WB_EINVAL, f"unknown {what} {name!r}; one of {', '.join(choices)}") from None


def _on(stream, call, *tensors):
    """``call()`` with ``stream`` current, so that its outputs belong to that
    stream; the inputs are kept until the stream's work is done."""
    import torch

    s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
    with torch.cuda.stream(s):
        out = call()
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(s)
    return out


def add_rms_norm(x, weight, residual=None, eps=1e-6, out_dtype=None, stream=None):
    """Root-mean-square norm of the rows of ``x + residual``:
    ``total * weight / sqrt(mean(total ** 2) + eps)``.

    Returns ``(out, scales, total)``. ``out_dtype`` is "f32", "bf16" or
    "f8e4m3" (default: x's own); ``scales`` is None unless it is "f8e4m3".
    ``total`` has the residual's type, and is None without one. The norm sees
    the sum before it is rounded."""
    if stream is not None:
        return _on(stream, lambda: add_rms_norm(x, weight, residual, eps, out_dtype), x, weight, residual)
    r = _args.add_rms_norm(_address("wb_add_rms_norm"), x, weight, residual, eps, _type(out_dtype, DTYPES, "out_dtype"),
                           *_here())
    return r if type(r) is tuple else _refused(r)


Routing = collections.namedtuple("Routing", "experts gates positions tokens counts offsets loss routed mask renormalize")
Routing.__doc__ = """Where the rows of a batch go (T rows, E experts, k choices).

experts [T, k]: the chosen experts, largest logit first, -1 where there is none; gates [T, k]: their weights;
positions [T, k]: each choice's place in expert order (-1: none); tokens [T * k]: the row at each place (-1 past the
last); counts [E]: places of each expert; offsets [E + 1]: its first place, and the number of places; loss: balance
loss; routed [1]: rows that were sent anywhere. mask and renormalize are as given."""


def route(logits, k, mask=None, renormalize=True, stream=None):
    """Send each row of ``logits`` [T, E] to its k largest experts (ties to the
    lower one). Gates are the softmax at the chosen, divided by their sum if
    ``renormalize``. Rows whose ``mask`` is 0, or that have no logit above
    -inf, go nowhere. The balance loss is
    ``E / (k n^2) * sum_e counts[e] * sum_t p[t, e]`` over the n rows routed.

    Returns a Routing; ``gates`` and ``loss`` are differentiable if ``logits``
    requires a gradient, once: a second derivative raises WbError."""
    if stream is not None:
        return _on(stream, lambda: route(logits, k, mask, renormalize), logits, mask)
    if getattr(logits, "requires_grad", False) and _grad_enabled():
        return Routing(*_differentiable()(logits, k, mask, renormalize), mask, bool(renormalize))
    return Routing(*_route(logits, k, mask, renormalize), mask, bool(renormalize))


def route_backward(logits, routing, d_gates=None, d_loss=None, stream=None):
    """Gradient of ``logits`` from those of ``routing.gates`` [T, k] and
    ``routing.loss`` (float32 tensors; None: zero), in the logits' type. It has
    no gradient in turn: d_gates and d_loss that require one raise WbError."""
    if stream is not None:
        return _on(stream, lambda: route_backward(logits, routing, d_gates, d_loss), logits, d_gates, d_loss,
                   *routing[:9])
    return _backward(logits, routing.experts, routing.gates, routing.counts, routing.routed, routing.mask,
                     routing.renormalize, d_gates, d_loss)


def _route(logits, k, mask, renormalize):
    r = _args.route(_address("wb_route"), _address("wb_route_workspace"), logits, mask, k, bool(renormalize), *_here())
    return r if type(r) is tuple else _refused(r)


def _backward(logits, experts, gates, counts, routed, mask, renormalize, d_gates, d_loss):
    r = _args.route_backward(_address("wb_route_backward"), logits, mask, experts.shape[1], bool(renormalize), experts,
                             gates, counts, routed, d_gates, d_loss, *_here())
    return _refused(r) if isinstance(r, (str, int)) else r


def _grad_enabled():
    _here()
    return _torch.is_grad_enabled()


_apply = None


def _differentiable():
    global _apply
    if _apply is None:
        import torch

        class Last(torch.autograd.Function):
            """A gradient that depends on ``of``, which has no gradient itself: asking for one is an error."""

            @staticmethod
            def forward(ctx, d, *of):
                return d.clone()

            @staticmethod
            def backward(ctx, *_):
                raise WbError(WB_EUNSUPPORTED, "route's gradient has no gradient of its own")

        class Route(torch.autograd.Function):
            @staticmethod
            def forward(ctx, logits, k, mask, renormalize):
                out = _route(logits.detach(), k, mask, renormalize)
                experts, gates, positions, tokens, counts, offsets, _, routed = out
                ctx.save_for_backward(logits, mask, experts, gates, counts, routed)
                ctx.renormalize = renormalize
                ctx.mark_non_differentiable(experts, positions, tokens, counts, offsets, routed)
                return out

            @staticmethod
            def jvp(ctx, *_):
                raise WbError(WB_EINVAL, "logits has a forward-mode tangent, which the operators do not carry on")

            @staticmethod
            def backward(ctx, _e, d_gates, _p, _t, _c, _o, d_loss, _r):
                logits, mask, experts, gates, counts, routed = ctx.saved_tensors
                with torch.no_grad():
                    d = _backward(logits.detach(), experts, gates.detach(), counts, routed, mask,
                                  ctx.renormalize, d_gates.contiguous(), d_loss.contiguous())
                if torch.is_grad_enabled():  # create_graph
                    d = Last.apply(d, logits, d_gates, d_loss)
                return d, None, None, None

        _apply = Route.apply
    return _apply


def linear(x, weight, bias=None, *, x_scales=None, weight_scales=None, activation="none", gated=False, residual=None,
           out_dtype="bf16", stream=None):
    """``act(x @ weight.T + bias) + residual``; with ``gated``, where the
    weight's rows are [gate; up], ``act(gate) * up + residual``.

    x [T, K] and weight [N, K] are both bf16, or both fp8 with ``x_scales``
    [T, ceil(K / 128)] and ``weight_scales`` [ceil(N / 128), ceil(K / 128)].
    ``activation`` is "none", "silu" or "gelu" (by erf). Returns the result in
    ``out_dtype`` ("bf16", "f32"), or ``(values, scales)`` for "f8e4m3"."""
    if stream is not None:
        return _on(stream, lambda: linear(x, weight, bias, x_scales=x_scales, weight_scales=weight_scales,
                                          activation=activation, gated=gated, residual=residual, out_dtype=out_dtype),
                   x, weight, bias, x_scales, weight_scales, residual)
    return _linear(x, weight, None, None, x_scales, weight_scales, bias, residual, activation, gated, out_dtype)


def expert_linear(x, weight, offsets, tokens=None, bias=None, *, x_scales=None, weight_scales=None, activation="none",
                  gated=False, residual=None, out_dtype="bf16", stream=None):
    """``linear`` with stacked weights [E, N, K] (scales [E, ceil(N / 128),
    ceil(K / 128)], bias [E, N]): row p of the result is of the expert with
    ``offsets[e] <= p < offsets[e + 1]`` (int32 [E + 1]; a rank's slice of
    Routing.offsets) and comes from row ``tokens[p]`` of x (int32), or from
    row p without ``tokens``. Rows of no expert hold nothing in particular:
    the result is new memory that they are not written to."""
    if stream is not None:
        return _on(stream, lambda: expert_linear(x, weight, offsets, tokens, bias, x_scales=x_scales,
                                                 weight_scales=weight_scales, activation=activation, gated=gated,
                                                 residual=residual, out_dtype=out_dtype),
                   x, weight, offsets, tokens, bias, x_scales, weight_scales, residual)
    if offsets is None:
        raise WbError(WB_EINVAL, "offsets is None")
    return _linear(x, weight, offsets, tokens, x_scales, weight_scales, bias, residual, activation, gated, out_dtype)


def _linear(x, weight, offsets, tokens, x_scales, weight_scales, bias, residual, activation, gated, out_dtype):
    r = _args.linear(_address("wb_linear"), _address("wb_linear_workspace"), x, weight, offsets, tokens, x_scales, weight_scales, bias, residual,
                     _type(activation, ACTIVATIONS, "activation"), bool(gated), _type(out_dtype, DTYPES, "out_dtype"),
                     *_here())
    return _refused(r) if isinstance(r, (str, int)) else r


def combine(y, positions, gates, residual=None, span=None, out_dtype=None, stream=None):
    """``residual[t] + sum_i gates[t, i] * y[positions[t, i]]``, summed in
    fp32. Places outside y's rows are left out, and with ``span`` (int32: the
    slice of Routing.offsets of this rank's experts) those outside
    ``span[0] <= place < span[-1]``. ``out_dtype``: "bf16" or "f32" (default:
    y's own)."""
    if stream is not None:
        return _on(stream, lambda: combine(y, positions, gates, residual, span, out_dtype), y, positions, gates,
                   residual, span)
    r = _args.combine(_address("wb_combine"), y, positions, gates, residual, span, _type(out_dtype, DTYPES, "out_dtype"),
                      *_here())
    return _refused(r) if isinstance(r, (str, int)) else r
