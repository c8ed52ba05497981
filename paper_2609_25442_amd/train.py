"""Operators around an MoE layer at the trainer, each with its gradient: the
lookup of token embeddings (``embedding``), the layer norm of a residual sum
(``add_layer_norm``), rows sorted by expert and back (``dispatch``,
``collect``, with what ``route`` returns), and the activation with a checkpoint
in 8 bits (``activate``).

They are called as the operators of ``ops`` are: outputs are made with torch, the
kernels are enqueued on the stream (the current one by default), tensors are
float32 or bfloat16 in the memory of the current device with rows any distance
apart, and arguments that do not fit raise WbError. Where a tensor requires a
gradient and gradients are recorded, results are part of its graph, once: a
second derivative raises WbError, and so does a tensor with a forward-mode
tangent. The ``..._backward`` functions compute the same gradients without a graph, for
programs that keep none.

A stream that is being captured accumulates a leaf's gradient where the leaf's
living graphs do: these functions raise WbError while a graph recorded on another stream
is alive. Drop it, or capture the ``..._backward`` functions.
"""

from __future__ import annotations

import collections

from . import DTYPES, WB_EINVAL, WB_EUNSUPPORTED, WbError, _args
from .ops import ACTIVATIONS, _address, _differentiated, _here, _on, _refused, _type


def _result(r):
    return _refused(r) if isinstance(r, (str, int)) else r


def _code(dtype):
    """The library's number of a torch type; -1 for None."""
    import torch

    return {None: -1, torch.float32: 0, torch.bfloat16: 1}.get(dtype, 99)


def _rows(d):
    """A gradient as the kernels read it: torch hands out expanded and transposed ones too."""
    if d is None or d.dim() != 2:
        return d if d is None else d.contiguous()
    rows, cols = d.shape
    fits = (cols <= 1 or d.stride(1) == 1) and (rows <= 1 or d.stride(0) >= cols)
    return d if fits else d.contiguous()


_functions = None


def _graph():
    """The operators as parts of torch's graphs (made at the first use, as torch is imported late)."""
    global _functions
    if _functions is not None:
        return _functions
    import torch

    class Last(torch.autograd.Function):
        """A gradient that depends on ``of`` and has none itself: asking for one is an error."""

        @staticmethod
        def forward(ctx, d, *of):
            return d.clone()

        @staticmethod
        def backward(ctx, *_):
            raise WbError(WB_EUNSUPPORTED, "this operator's gradient has no gradient of its own")

    def last(grads, *of):
        if not torch.is_grad_enabled():  # else create_graph
            return grads
        of = [t for t in of if t is not None]
        return tuple(g if g is None else Last.apply(g, *of) for g in grads)

    class Function(torch.autograd.Function):
        @staticmethod
        def jvp(ctx, *_):
            raise WbError(WB_EINVAL, "an argument has a forward-mode tangent, which the operators do not carry on")

    def plain(t):
        return t.detach() if isinstance(t, torch.Tensor) else t

    class Embedding(Function):
        @staticmethod
        def forward(ctx, weight, tokens, scale, first, out_dtype):
            ctx.save_for_backward(tokens)
            ctx.more = weight.shape[0], scale, first, weight.dtype
            return _embedding(tokens, weight.detach(), scale, first, out_dtype)

        @staticmethod
        def backward(ctx, d_out):
            (tokens,), (rows, scale, first, dtype) = ctx.saved_tensors, ctx.more
            with torch.no_grad():
                d = _embedding_backward(_rows(d_out.detach()), tokens, rows, scale, first, _code(dtype))
            return *last((d,), d_out), None, None, None, None

    class AddLayerNorm(Function):
        @staticmethod
        def forward(ctx, x, weight, bias, residual, eps, center, out_dtype):
            ctx.set_materialize_grads(False)
            out, total, mean, inv = _add_layer_norm(plain(x), plain(weight), plain(bias), plain(residual), eps, center,
                                                    out_dtype)
            ctx.save_for_backward(x if residual is None else total, weight, mean, inv)
            ctx.types = x.dtype, None if residual is None else residual.dtype, None if bias is None else bias.dtype
            ctx.mark_non_differentiable(*(t for t in (mean, inv) if t is not None))
            return out, total, mean, inv

        @staticmethod
        def backward(ctx, d_out, d_total, *_):
            total, weight, mean, inv = ctx.saved_tensors
            of_x, of_residual, of_bias = ctx.types
            need = ctx.needs_input_grad
            if d_out is None:  # only the sum went on
                return None if d_total is None else d_total.to(of_x), None, None, d_total, None, None, None
            with torch.no_grad():
                w = weight.dtype if need[1] else of_bias if need[2] else None
                d_x, d_residual, d_weight, d_bias = _add_layer_norm_backward(
                    _rows(d_out.detach()), total.detach(), weight.detach(), _rows(plain(d_total)), mean, inv, of_x, of_residual,
                    w, of_bias if need[2] else None)
            grads = last((d_x, d_weight if need[1] else None, d_bias, d_residual), d_out, d_total, total, weight)
            return *grads, None, None, None

    class Dispatch(Function):
        @staticmethod
        def forward(ctx, x, positions, tokens, span):
            ctx.save_for_backward(positions, tokens, span)
            ctx.type = x.dtype
            return _dispatch(x.detach(), positions, tokens, span)

        @staticmethod
        def backward(ctx, d_rows):
            with torch.no_grad():
                d = _dispatch_backward(_rows(d_rows.detach()), *ctx.saved_tensors, _code(ctx.type))
            return *last((d,), d_rows), None, None, None

    class Collect(Function):
        @staticmethod
        def forward(ctx, y, gates, residual, positions, tokens, span, out_dtype):
            out = _collect(plain(y), positions, tokens, plain(gates), plain(residual), span, out_dtype)
            need_y, need_gates = ctx.needs_input_grad[:2]
            # y is read for the gates' gradient alone, and none of them for the residual's
            kept = (y if need_gates else None, gates, positions, tokens, span) if need_y or need_gates else ()
            ctx.save_for_backward(*kept)
            ctx.types = y.dtype, None if residual is None else residual.dtype
            return out

        @staticmethod
        def backward(ctx, d_out):
            need_y, need_gates = ctx.needs_input_grad[:2]
            of_y, of_residual = ctx.types
            d_y = d_gates = None
            if need_y or need_gates:
                y, gates, positions, tokens, span = ctx.saved_tensors
                with torch.no_grad():
                    d_y, d_gates = _collect_backward(_rows(d_out.detach()), plain(y) if need_gates else None, positions, tokens,
                                                     gates.detach(), span, of_y if need_y else None)
                d_y, d_gates = last((d_y, d_gates), d_out, y, gates)
            d_residual = d_out.to(of_residual) if ctx.needs_input_grad[2] else None
            return d_y, d_gates, d_residual, None, None, None, None

    class Activate(Function):
        @staticmethod
        def forward(ctx, x, activation, gated, checkpoint, out_dtype):
            # else torch makes zeros of the codes' and the scales' shapes, as gradients that nothing reads
            ctx.set_materialize_grads(False)
            out, codes, scales = _activate(x.detach(), activation, gated, checkpoint, out_dtype)
            ctx.save_for_backward(codes if checkpoint else x, scales)
            ctx.more = activation, gated, x.dtype
            if not checkpoint:
                return out, None, None
            ctx.mark_non_differentiable(codes, scales)
            return out, codes, scales

        @staticmethod
        def backward(ctx, d_out, *_):
            if d_out is None:
                return (None,) * 5
            saved, scales = ctx.saved_tensors
            with torch.no_grad():
                d = _activate_backward(_rows(d_out.detach()), saved.detach(), scales, *ctx.more)
            return *last((d,), d_out, saved), None, None, None, None

    _functions = dict(embedding=Embedding.apply, add_layer_norm=AddLayerNorm.apply, dispatch=Dispatch.apply,
                      collect=Collect.apply, activate=Activate.apply)
    return _functions


# ---- embeddings --------------------------------------------------------------------------------


def embedding(tokens, weight, scale=1.0, first=0, out_dtype=None, stream=None):
    """``scale * weight[tokens - first]`` for token ids (int32 or int64, of any
    shape, contiguous), [*tokens.shape, cols]; zeros where that is no row of
    weight [V, cols]: a rank with a part of the vocabulary gives its first row's
    id, and the parts' results add up. ``out_dtype`` is "f32" or "bf16"
    (default: the weight's own).

    Differentiable in weight: row v's gradient is ``scale`` times the sum of the
    results' gradients where ``tokens - first == v``, in an order that the call's
    tokens fix."""
    if stream is not None:
        return _on(stream, lambda: embedding(tokens, weight, scale, first, out_dtype), tokens, weight)
    if _differentiated(weight):
        return _graph()["embedding"](weight, tokens, scale, first, out_dtype)
    return _embedding(tokens, weight, scale, first, out_dtype)


def embedding_backward(d_out, tokens, rows, scale=1.0, first=0, out_dtype=None, stream=None):
    """Gradient of a weight of ``rows`` rows from that of ``embedding``'s result
    [*tokens.shape, cols], in ``out_dtype`` ("f32" or "bf16"; default: d_out's own)."""
    if stream is not None:
        return _on(stream, lambda: embedding_backward(d_out, tokens, rows, scale, first, out_dtype), d_out, tokens)
    return _embedding_backward(d_out, tokens, rows, scale, first, _type(out_dtype, DTYPES, "out_dtype"))


def _embedding(tokens, weight, scale, first, out_dtype):
    return _result(_args.embedding(_address("wb_embedding"), tokens, weight, scale, first,
                                   _type(out_dtype, DTYPES, "out_dtype"), *_here()))


def _embedding_backward(d_out, tokens, rows, scale, first, type_):
    return _result(_args.embedding_backward(_address("wb_embedding_backward"), _address("wb_embedding_backward_workspace"),
                                            d_out, tokens, rows, scale, first, type_, *_here()))


# ---- layer norm --------------------------------------------------------------------------------

Normed = collections.namedtuple("Normed", "out total mean inv x_type residual_type bias_type")
Normed.__doc__ = """What ``add_layer_norm`` returns, and its gradient reads (T rows).

out: the normed rows; total: the sum that was normed, as it is kept (x itself without a residual); mean [T] (None:
not centred) and inv [T]: each row's statistics; x_type, residual_type, bias_type: the arguments' torch types, None
for an absent one."""

NormGradient = collections.namedtuple("NormGradient", "x residual weight bias")
NormGradient.__doc__ = """Gradients of ``add_layer_norm``'s arguments, each in its argument's type; None for an
absent one. x and residual have the same one, one tensor where their types are alike."""


def add_layer_norm(x, weight, bias=None, residual=None, eps=1e-5, center=True, out_dtype=None, stream=None):
    """Layer norm of the rows of ``total = x + residual``:
    ``(total - mean) / sqrt(var + eps) * weight + bias``, or without ``center``
    ``total / sqrt(mean(total ** 2) + eps) * weight + bias``.

    Returns a Normed. ``total`` has the residual's type and, unlike
    ``add_rms_norm``'s, is what the norm sees: the gradient reads it again.
    ``out_dtype`` is "f32" or "bf16" (default: x's own). ``out`` and ``total``
    are differentiable in x, weight, bias and residual."""
    if stream is not None:
        return _on(stream, lambda: add_layer_norm(x, weight, bias, residual, eps, center, out_dtype), x, weight, bias,
                   residual)
    if _differentiated(x, weight, bias, residual):
        out, total, mean, inv = _graph()["add_layer_norm"](x, weight, bias, residual, eps, center, out_dtype)
    else:
        out, total, mean, inv = _add_layer_norm(x, weight, bias, residual, eps, center, out_dtype)
    if total is None:
        return Normed(out, x, mean, inv, x.dtype, None, None if bias is None else bias.dtype)
    return Normed(out, total, mean, inv, x.dtype, total.dtype, None if bias is None else bias.dtype)


def add_layer_norm_backward(d_out, normed, weight, d_total=None, stream=None):
    """The arguments' NormGradient from the gradients of ``normed.out`` and, where
    it went on elsewhere, of ``normed.total`` (None: zero)."""
    if stream is not None:
        return _on(stream, lambda: add_layer_norm_backward(d_out, normed, weight, d_total), d_out, weight, d_total,
                   *normed[1:4])
    return NormGradient(*_add_layer_norm_backward(d_out, normed.total, weight, d_total, normed.mean, normed.inv,
                                                  normed.x_type, normed.residual_type, getattr(weight, "dtype", None),
                                                  normed.bias_type))


def _add_layer_norm(x, weight, bias, residual, eps, center, out_dtype):
    return _result(_args.add_layer_norm(_address("wb_add_layer_norm"), x, weight, bias, residual, eps, bool(center),
                                        _type(out_dtype, DTYPES, "out_dtype"), *_here()))


def _add_layer_norm_backward(d_out, total, weight, d_total, mean, inv, x_type, residual_type, weight_type, bias_type):
    return _result(_args.add_layer_norm_backward(
        _address("wb_add_layer_norm_backward"), _address("wb_add_layer_norm_backward_workspace"), d_out, total, weight,
        d_total, mean, inv, _code(x_type), _code(residual_type), _code(weight_type), _code(bias_type), *_here()))


# ---- rows by expert and back -------------------------------------------------------------------


def dispatch(x, routing, span=None, stream=None):
    """x's rows [T, cols] in expert order, [T * k, cols] in x's type: row p is
    ``x[routing.tokens[p]]``. Rows past the last place are zeros, and with
    ``span`` (int32: the slice of ``routing.offsets`` of this rank's experts)
    those outside ``span[0] <= p < span[-1]``. Differentiable in x."""
    if stream is not None:
        return _on(stream, lambda: dispatch(x, routing, span), x, routing.positions, routing.tokens, span)
    if _differentiated(x):
        return _graph()["dispatch"](x, routing.positions, routing.tokens, span)
    return _dispatch(x, routing.positions, routing.tokens, span)


def dispatch_backward(d_rows, routing, span=None, out_dtype=None, stream=None):
    """Gradient of x from that of ``dispatch``'s rows: the sum of a row's places,
    in ``out_dtype`` ("f32" or "bf16"; default: d_rows' own)."""
    if stream is not None:
        return _on(stream, lambda: dispatch_backward(d_rows, routing, span, out_dtype), d_rows, routing.positions,
                   routing.tokens, span)
    return _dispatch_backward(d_rows, routing.positions, routing.tokens, span, _type(out_dtype, DTYPES, "out_dtype"))


def collect(y, routing, gates=None, residual=None, span=None, out_dtype=None, stream=None):
    """``residual[t] + sum_i gates[t, i] * y[routing.positions[t, i]]``: what
    ``combine`` computes, differentiable in y [T * k, cols], gates (default:
    ``routing.gates``) and residual. ``span`` and ``out_dtype`` as there.
    Choices whose place ``routing.tokens`` gives to another row, or that name a
    place again, are left out, as they are by ``dispatch``."""
    if stream is not None:
        return _on(stream, lambda: collect(y, routing, gates, residual, span, out_dtype), y, routing.positions,
                   routing.tokens, routing.gates, gates, residual, span)
    gates = routing.gates if gates is None else gates
    if _differentiated(y, gates, residual):
        return _graph()["collect"](y, gates, residual, routing.positions, routing.tokens, span, out_dtype)
    return _collect(y, routing.positions, routing.tokens, gates, residual, span, out_dtype)


def collect_backward(d_out, y, routing, gates=None, span=None, stream=None):
    """Gradients (of y, of the gates) from that of ``collect``'s result; the
    residual's is d_out. Rows of y that no token has get zeros, and so do gates
    of choices that were left out."""
    if stream is not None:
        return _on(stream, lambda: collect_backward(d_out, y, routing, gates, span), d_out, y, routing.positions,
                   routing.tokens, routing.gates, gates, span)
    return _collect_backward(d_out, y, routing.positions, routing.tokens, routing.gates if gates is None else gates, span,
                             getattr(y, "dtype", None))


def _dispatch(x, positions, tokens, span):
    return _result(_args.dispatch(_address("wb_dispatch"), x, positions, tokens, span, *_here()))


def _dispatch_backward(d_rows, positions, tokens, span, type_):
    return _result(_args.dispatch_backward(_address("wb_dispatch_backward"), d_rows, positions, tokens, span, type_, *_here()))


def _collect(y, positions, tokens, gates, residual, span, out_dtype):
    return _result(_args.collect(_address("wb_collect"), y, positions, tokens, gates, residual, span,
                                 _type(out_dtype, DTYPES, "out_dtype"), *_here()))


def _collect_backward(d_out, y, positions, tokens, gates, span, y_type):
    return _result(_args.collect_backward(_address("wb_combine_backward"), d_out, y, positions, tokens, gates, span,
                                          _code(y_type), *_here()))


# ---- activation --------------------------------------------------------------------------------

Activated = collections.namedtuple("Activated", "out saved scales activation gated x_type")
Activated.__doc__ = """What ``activate`` returns, and its gradient reads.

out: the result; saved: x itself, or its codes (float8_e4m3fn) with their scales [T, one per 128 columns of each
half]; activation and gated as given; x_type: x's torch type."""


def activate(x, activation="silu", gated=False, checkpoint=False, out_dtype=None, stream=None):
    """``act(x)``, or with ``gated``, where x's columns are [gate; up],
    ``act(gate) * up``. ``activation`` is "none", "silu" or "gelu" (by erf).

    Returns an Activated; ``out`` ("f32" or "bf16"; default: x's own) is
    differentiable in x. With ``checkpoint`` the graph keeps x in 8 bits (E4M3
    with a scale per row and 128 columns of each half) in place of x, and the
    gradient is taken at the values that these stand for; the result is that of x."""
    if stream is not None:
        return _on(stream, lambda: activate(x, activation, gated, checkpoint, out_dtype), x)
    if _differentiated(x):
        out, codes, scales = _graph()["activate"](x, activation, gated, checkpoint, out_dtype)
    else:
        out, codes, scales = _activate(x, activation, gated, checkpoint, out_dtype)
    return Activated(out, codes if checkpoint else x, scales, activation, bool(gated), x.dtype)


def activate_backward(d_out, activated, stream=None):
    """Gradient of x, in its type, from that of ``activated.out``."""
    if stream is not None:
        return _on(stream, lambda: activate_backward(d_out, activated), d_out, *activated[1:3])
    return _activate_backward(d_out, activated.saved, activated.scales, activated.activation, activated.gated,
                              activated.x_type)


def _activate(x, activation, gated, checkpoint, out_dtype):
    return _result(_args.activate(_address("wb_activate"), x, _type(activation, ACTIVATIONS, "activation"), bool(gated),
                                  bool(checkpoint), _type(out_dtype, DTYPES, "out_dtype"), *_here()))


def _activate_backward(d_out, saved, scales, activation, gated, x_type):
    return _result(_args.activate_backward(_address("wb_activate_backward"), d_out, saved, scales,
                                           _type(activation, ACTIVATIONS, "activation"), bool(gated), _code(x_type), *_here()))
