"""A dropless MoE layer: tokens sorted by expert and back with their weights, the experts' products on the sorted rows, and the
gradients of all of it, the router's among them.

The functions allocate their outputs (and the workspace, from torch's allocator on the current stream) and call the entry
points of ``binding``; all arithmetic runs in the CUDA library.  ``stream`` is as in ``block``.  ``moe_layer`` is the
differentiable layer; ``RouteSort``, ``ExpertFFN`` and ``Unsort`` are its parts.
"""
from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .block import _F32, _count, _flat, _here, _rows, _shape, _under, _want_rows, _empty_strided_cuda

_ACTS = {None: B.ACT_NONE, "none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}
_BF, _I32 = torch.bfloat16, torch.int32


class Order(NamedTuple):
    """Where the K * T assignments v = c * T + t (choice c of token t) lie once sorted by expert: expert e's rows are
    [offsets[e], offsets[e + 1]), ``slot`` [K][T] is the row of an assignment (-1: not routed) and ``inv`` [K * T] the
    assignment of a row (-1 behind the last group).  ``load`` [E] counts the tokens by their first choice."""
    offsets: torch.Tensor
    slot: torch.Tensor
    inv: torch.Tensor
    load: Optional[torch.Tensor] = None


@lru_cache(maxsize=1024)
def _sort_grad_bytes(shape_key) -> int:
    T, H, E, dtype, _ = shape_key
    return B.locmoe_sort_grad_bytes(_shape(T, H, E, dtype))


@lru_cache(maxsize=1024)
def _linear_plan(R: int, H: int, E: int, N: int, grad: bool, device: int):
    _count(N)
    shape = _shape(R, H, E, _BF)
    return shape, B.locmoe_expert_linear_bytes(shape, N, grad)


def _act(act) -> int:
    try:
        return _ACTS[act]
    except (KeyError, TypeError):
        raise ValueError("act: expected one of none, relu, gelu, silu, got %r" % (act,)) from None


def _matrix(t: torch.Tensor, name: str):
    if t.dim() != 2:
        raise ValueError("%s: expected a matrix, got %s" % (name, tuple(t.shape)))
    return t.shape


def _slots(order: Order, T: int) -> int:
    """K of an order for T tokens."""
    s = order.slot.shape
    if len(s) != 2 or s[1] != T:
        raise ValueError("order.slot: expected [K][%d], got %s" % (T, tuple(s)))
    return s[0]


def _on_current(t, name: str) -> None:
    """For the router's calls, whose binding does not compare devices."""
    if t is not None and (not t.is_cuda or t.get_device() != torch.cuda.current_device()):
        raise ValueError("%s: on %s, which is not the current CUDA device" % (name, t.device))


def _want_shape(t, shape: tuple, name: str) -> None:
    if t is not None and t.shape != shape:
        raise ValueError("%s: expected %s, got %s" % (name, shape, tuple(t.shape)))


def sort_rows(x, idx_k, E: int, want_load=False, want_rows=True, stream=None):
    """Sorts the choices idx_k [K][T] (int32; outside [0, E): not routed) by expert: ``(xs, order)``, xs [K * T][H] the rows of
    x [T][H] (bf16 or fp32) in that order, zeros behind the last group.  xs is None without ``want_rows``."""
    if stream is not None:
        with _under(stream):
            return sort_rows(x, idx_k, E, want_load, want_rows)
    T, H = _matrix(x, "x")
    if idx_k.dim() != 2 or idx_k.shape[1] != T:
        raise ValueError("idx_k: expected [K][%d], got %s" % (T, tuple(idx_k.shape)))
    K = idx_k.shape[0]
    shape = _shape(T, H, E, x.dtype)
    _here(x, "x")
    _count(K * T)
    order = Order(_flat(E + 1, _I32), _rows(K, T, _I32), _flat(K * T, _I32), _flat(E, _I32) if want_load else None)
    xs = _rows(K * T, H, x.dtype) if want_rows else None
    if T == 0:
        order.offsets.zero_()
        if want_load:
            order.load.zero_()
        return xs, order
    B.locmoe_sort(shape, K, idx_k, order.offsets, order.slot, order.inv, order.load, x if want_rows else None, xs)
    return xs, order


def sort_rows_grad(dxs, order: Order, x=None, idx_k=None, dw=None, eps=None, dp=None, want_deps=True, stream=None):
    """Gradient of ``sort_rows`` towards the tokens from dxs [K * T][H]: ``(dx, deps)``.

    With the tokens x [T][H] the router's own gradient is added: ``dw`` [K][T] is the gradient of the chosen scores (with
    ``idx_k``), ``dp`` [E] that of every token's probabilities, ``eps`` [E] the bias the router ran with; deps [E] is then the
    gradient of eps, else None.  A group mean that is NaN counts as 0, as in the forward pass.  dxs may be None with x."""
    if stream is not None:
        with _under(stream):
            return sort_rows_grad(dxs, order, x, idx_k, dw, eps, dp, want_deps)
    if dxs is None and x is None:
        raise ValueError("dxs, x: one of them is needed")
    if x is None and not (dw is eps is dp is None):
        raise ValueError("x: needed for the router's gradient")
    if dw is not None and idx_k is None:
        raise ValueError("idx_k: needed with dw")
    E = order.offsets.numel() - 1
    like = x if x is not None else dxs
    n, H = _matrix(like, "x" if x is not None else "dxs")
    T = order.slot.shape[-1]
    K = _slots(order, T)
    if x is not None and n != T:
        raise ValueError("x: expected %d rows, got %d" % (T, n))
    if dxs is not None:
        if dxs.dtype != like.dtype:
            raise TypeError("dxs: expected %s, got %s" % (like.dtype, dxs.dtype))
        _want_rows(dxs, K * T, H, "dxs")
    _want_shape(dw, (K, T), "dw")
    if dw is not None:
        _want_shape(idx_k, (K, T), "idx_k")
    _want_shape(eps, (E,), "eps")
    _want_shape(dp, (E,), "dp")
    shape = _shape(T, H, E, like.dtype)
    _here(like, "rows")
    dx = _rows(T, H, like.dtype)
    deps = _flat(E, _F32) if want_deps and x is not None else None
    if T == 0:
        if deps is not None:
            deps.zero_()
        return dx, deps
    ws = _flat(_sort_grad_bytes((T, H, E, like.dtype, torch.cuda.current_device())), torch.uint8) if deps is not None else None
    B.locmoe_sort_grad(shape, K, order.slot, dx, dxs, x, eps, idx_k if dw is not None else None, dw, dp, deps, ws)
    return dx, deps


def unsort_rows(y, order: Order, w_k=None, residual=None, stream=None):
    """out[t] = residual[t] + sum over a token's choices of w_k[c][t] * y[slot[c][t]]: y [K * T][H], out [T][H]."""
    if stream is not None:
        with _under(stream):
            return unsort_rows(y, order, w_k, residual)
    n, H = _matrix(y, "y")
    T = order.slot.shape[-1]
    K = _slots(order, T)
    _want_rows(y, K * T, H, "y")
    _want_shape(w_k, (K, T), "w_k")
    _want_shape(residual, (T, H), "residual")
    shape = _shape(T, H, order.offsets.numel() - 1, y.dtype)
    _here(y, "y")
    out = _rows(T, H, y.dtype)
    if T > 0:
        B.locmoe_unsort(shape, K, y, order.slot, out, w_k, residual)
    return out


def unsort_rows_grad(dout, order: Order, w_k=None, y=None, want_dy=True, stream=None):
    """Gradient of ``unsort_rows`` from dout [T][H]: ``(dy, dw)``, dw None without y, dy None where it is not wanted.  The gradient
    of the residual is dout."""
    if stream is not None:
        with _under(stream):
            return unsort_rows_grad(dout, order, w_k, y, want_dy)
    if y is None and not want_dy:
        raise ValueError("y, want_dy: nothing is asked for")
    T, H = _matrix(dout, "dout")
    K = _slots(order, T)
    if y is not None:
        if y.dtype != dout.dtype:
            raise TypeError("y: expected %s, got %s" % (dout.dtype, y.dtype))
        _want_rows(y, K * T, H, "y")
    _want_shape(w_k, (K, T), "w_k")
    shape = _shape(T, H, order.offsets.numel() - 1, dout.dtype)
    _here(dout, "dout")
    dy = _rows(K * T, H, dout.dtype) if want_dy else None
    dw = _rows(K, T, _F32) if y is not None else None
    if T > 0:
        B.locmoe_unsort_grad(shape, K, dout, order.offsets, order.slot, y, w_k, dy, dw)
    return dy, dw


def _linear_sizes(rows, w, offsets, name: str, out_side: bool):
    R, n = _matrix(rows, name)
    if w.dim() != 3:
        raise ValueError("w: expected [E][OUT][IN], got %s" % (tuple(w.shape),))
    E, N, H = w.shape
    if n != (N if out_side else H):
        raise ValueError("%s %s and w %s do not belong together" % (name, tuple(rows.shape), tuple(w.shape)))
    _want_shape(offsets, (E + 1,), "offsets")
    return R, H, E, N


def expert_linear(x, w, offsets, bias=None, act=None, residual=None, want_z=False, stream=None):
    """y = act(z) + residual, z[r] = w[e] x[r] + bias[e] for the rows [offsets[e], offsets[e + 1]) of every expert e.

    x [R][IN], w [E][OUT][IN], residual [R][OUT] bf16, bias [E][OUT] fp32; act one of none, relu, gelu, silu.  Returns ``(y, z)``,
    z (bf16, for the gradient) None without ``want_z``; rows of no group (behind the last, or before the first where offsets is a
    slice for a part of the experts) are zero in both."""
    if stream is not None:
        with _under(stream):
            return expert_linear(x, w, offsets, bias, act, residual, want_z)
    R, H, E, N = _linear_sizes(x, w, offsets, "x", False)
    code = _act(act)
    _want_shape(bias, (E, N), "bias")
    _want_shape(residual, (R, N), "residual")
    _here(x, "x")
    if R > 0:
        shape, n = _linear_plan(R, H, E, N, False, torch.cuda.current_device())
    y = _rows(R, N, _BF)
    z = _rows(R, N, _BF) if want_z else None
    if R > 0:
        B.locmoe_expert_linear(shape, N, x, w, offsets, y, _flat(n, torch.uint8), bias, residual, z, code)
    return y, z


def expert_linear_grad(dy, x, w, offsets, z=None, act=None, want_dx=True, want_dw=True, want_db=False, dw_dtype=None, stream=None):
    """Gradient of the products from dy [R][OUT], the gradient of z: ``(dx, dw, db)``, each None when not wanted.

    With ``z`` [R][IN], what the rows x = act(z) were made of, dx is the gradient of that z: it has gone through the activation
    before this product.  dw [E][OUT][IN] is in ``dw_dtype`` (bf16 or fp32, by default w's), db [E][OUT] in fp32.  Rows of
    no group: zeros in dx, no part of dw and db.  x may be None without ``want_dw``."""
    if stream is not None:
        with _under(stream):
            return expert_linear_grad(dy, x, w, offsets, z, act, want_dx, want_dw, want_db, dw_dtype)
    R, H, E, N = _linear_sizes(dy, w, offsets, "dy", True)
    code = _act(act)
    if not (want_dx or want_dw or want_db):
        raise ValueError("want_dx, want_dw, want_db: nothing is asked for")
    if want_dw and x is None:
        raise ValueError("x: needed for dw")
    if z is not None and code == B.ACT_NONE:
        raise ValueError("act: needed with z")
    _want_shape(x, (R, H), "x")
    _want_shape(z, (R, H), "z")
    if dw_dtype is None:
        dw_dtype = w.dtype if want_dw else _BF
    if dw_dtype not in (_BF, _F32):
        raise TypeError("dw_dtype: expected bfloat16 or float32, got %s" % (dw_dtype,))
    _here(dy, "dy")
    if R > 0:
        shape, n = _linear_plan(R, H, E, N, True, torch.cuda.current_device())
    dx = _rows(R, H, _BF) if want_dx else None
    dw = _empty_strided_cuda((E, N, H), (N * H, H, 1), dw_dtype) if want_dw else None
    db = _rows(E, N, _F32) if want_db else None
    if R == 0:
        for t in (dw, db):
            if t is not None:
                t.zero_()
        return dx, dw, db
    ws = _flat(n, torch.uint8) if want_dx or want_dw else None
    B.locmoe_expert_linear_grad(shape, N, dy, offsets, x if want_dw else None, w if want_dx else None, z if want_dx else None, dx, dw, db, code, ws)
    return dx, dw, db


# ---- the differentiable layer ----

def _dense(t):
    return None if t is None else t.contiguous()


# A leaf's gradient is added up on the stream that the node for it was made on, by whichever operator came first, and the node
# lives as long as any graph that reached it.  If that was the default stream, which no capture can take in, a captured backward
# pass through it spoils the capture and can end the process.  So a captured backward pass asks each node for its stream and
# refuses before any gradient is sent there.  The node says it to a hook of its leaf only: a pass that sends it nothing reaches
# the hook on that stream, and ends there, before anything is launched or waited for.
class _Found(Exception):
    pass


class _Nothing(torch.autograd.Function):
    """A number of the host's that depends on a tensor and gives it no gradient."""

    @staticmethod
    def forward(ctx, t):
        return torch.zeros(())

    @staticmethod
    def backward(ctx, g):
        return None


def _leaf_stream(leaf) -> int:
    """The stream (a raw handle, 0: the default stream) that gradients of this leaf are added up on."""
    if not leaf.requires_grad:      # any more: its node cannot be asked
        return 0
    found = []

    def hook(_):
        found.append(B._raw_stream(leaf.get_device()))
        raise _Found
    with torch.enable_grad():
        out = _Nothing.apply(leaf)
    others = dict(leaf._backward_hooks or {})                   # are for gradients
    if others:
        leaf._backward_hooks.clear()
    handle = leaf.register_hook(hook)
    try:
        out.backward()
    except _Found:
        pass
    finally:
        handle.remove()
        leaf._backward_hooks.update(others)
    return found[0]


def _check_capture(ctx) -> None:
    if not torch.cuda.is_current_stream_capturing():
        return
    for node, _ in ctx.next_functions:
        if node is not None and type(node).__name__ == "AccumulateGrad" and _leaf_stream(node.variable) == 0:
            raise RuntimeError("a captured backward pass: a graph of the same leaves that was built on the default stream is still "
                               "alive; drop its outputs first, or build it on another stream")


class RouteSort(torch.autograd.Function):
    """``RouteSort.apply(x, eps, E, K, alpha) -> (xs, w_k, aux, idx_k, offsets, slot, inv)``: the router and the tokens in the
    order of its choices.  Differentiable in x and eps, once; aux is the load-balance loss alpha * E * sum f_i P_i (None with
    alpha = 0)."""

    @staticmethod
    def forward(ctx, x, eps, E, K=1, alpha=0.0):
        T, H = _matrix(x, "x")
        if not 1 <= K <= min(8, E):
            raise ValueError("K: expected 1 to %d, got %d" % (min(8, E), K))
        _on_current(x, "x")
        _on_current(eps, "eps")
        _want_shape(eps, (E,), "eps")
        ctx.set_materialize_grads(False)
        idx_k, w_k, aux, f = _rows(K, T, _I32), _rows(K, T, _F32), None, None
        if T > 0:
            shape = _shape(T, H, E, x.dtype)
            idx, gate_w = (idx_k[0], w_k[0]) if K == 1 else (_flat(T, _I32), _flat(T, _F32))
            probs = _rows(T, E, _F32) if K > 1 else None
            part = _flat(B.GATE_PARTIAL_ROWS * E, _F32) if alpha else None
            p_rows = B.locmoe_gate_ex(shape, x, idx, gate_w, _flat(T, _F32), eps=eps, probs=probs, p_part=part)
            if K > 1:
                B.locmoe_topk_select(shape, probs, idx, gate_w, K, idx_k, w_k)
        xs, order = sort_rows(x, idx_k, E, want_load=bool(alpha))
        if alpha:
            aux = torch.zeros((), dtype=_F32, device=x.device)
            f = torch.zeros(E, dtype=_F32, device=x.device)
            if T > 0:
                B.locmoe_aux_loss_partial(shape, part, p_rows, order.load, alpha, f, _flat(E, _F32), aux)
        ctx.alpha = alpha
        ctx.save_for_backward(x, eps, idx_k, order.offsets, order.slot, order.inv, f)
        ctx.mark_non_differentiable(idx_k, order.offsets, order.slot, order.inv)
        return xs, w_k, aux, idx_k, order.offsets, order.slot, order.inv

    @staticmethod
    @once_differentiable
    def backward(ctx, dxs, dw, daux, *_):
        _check_capture(ctx)
        x, eps, idx_k, offsets, slot, inv, f = ctx.saved_tensors
        if dxs is None and dw is None and daux is None:
            return (None,) * 5
        if x.shape[0] == 0:
            return torch.zeros_like(x), torch.zeros_like(eps) if ctx.needs_input_grad[1] else None, None, None, None
        dp = None
        if daux is not None:
            dp = f * (daux * (ctx.alpha * f.numel() / x.shape[0]))
        router = dw is not None or dp is not None
        dx, deps = sort_rows_grad(_dense(dxs), Order(offsets, slot, inv), x if router else None, idx_k, _dense(dw), eps if router else None, dp,
                                  want_deps=ctx.needs_input_grad[1])
        if deps is None and ctx.needs_input_grad[1]:
            deps = torch.zeros_like(eps)
        return dx, deps, None, None, None


class ExpertFFN(torch.autograd.Function):
    """``ExpertFFN.apply(xs, w_in, w_out, b_in, b_out, offsets, act) -> y``: w_out act(w_in x + b_in) + b_out on sorted rows, one
    expert's weights for each group.  Differentiable in its first five arguments, once; what is kept is the first product's
    output before and after the activation."""

    @staticmethod
    def forward(ctx, xs, w_in, w_out, b_in, b_out, offsets, act="gelu"):
        a, z = expert_linear(xs, w_in, offsets, b_in, act, want_z=_act(act) != B.ACT_NONE)
        y, _ = expert_linear(a, w_out, offsets, b_out)
        ctx.act = act
        ctx.save_for_backward(xs, w_in, w_out, b_in, b_out, offsets, a, z)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        _check_capture(ctx)
        xs, w_in, w_out, b_in, b_out, offsets, a, z = ctx.saved_tensors
        need = ctx.needs_input_grad
        dy = dy.contiguous()
        first = need[0] or need[1] or need[3]
        dz = dw_out = db_out = dxs = dw_in = db_in = None
        if first or need[2] or need[4]:
            dz, dw_out, db_out = expert_linear_grad(dy, a, w_out, offsets, z, ctx.act if z is not None else None, want_dx=first, want_dw=need[2],
                                                    want_db=need[4])
        if first:
            dxs, dw_in, db_in = expert_linear_grad(dz, xs, w_in, offsets, want_dx=need[0], want_dw=need[1], want_db=need[3])
        return dxs, dw_in, dw_out, db_in, db_out, None, None


class Unsort(torch.autograd.Function):
    """``Unsort.apply(y, w_k, residual, offsets, slot, inv) -> out``, differentiable in its first three arguments, once."""

    @staticmethod
    def forward(ctx, y, w_k, residual, offsets, slot, inv):
        ctx.save_for_backward(y, w_k, offsets, slot, inv)
        return unsort_rows(y, Order(offsets, slot, inv), w_k, residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        _check_capture(ctx)
        y, w_k, offsets, slot, inv = ctx.saved_tensors
        need = ctx.needs_input_grad
        dy = dw = None
        if need[0] or need[1]:
            dy, dw = unsort_rows_grad(dout.contiguous(), Order(offsets, slot, inv), w_k, y if need[1] else None, want_dy=need[0])
        return dy, dw, dout if need[2] else None, None, None, None


def moe_layer(x, w_in, w_out, K=1, b_in=None, b_out=None, eps=None, act="gelu", residual=None, alpha=0.0):
    """The MoE layer without a capacity: out[t] = residual[t] + sum over the K best experts of score * FFN_e(x[t]).

    x [T][H], w_in [E][F][H], w_out [E][H][F] bf16; b_in [E][F], b_out [E][H] and eps [E] (the router's bias) fp32, or None.
    Returns ``(out, aux)``, aux the load-balance loss with alpha > 0, else None.  Differentiable in all tensors.  Every token is
    routed; a padded batch goes through the functions one by one (``sort_rows`` takes -1 for a token that is not).

    Forward and backward can be captured into a CUDA graph; no graph of the same leaves that was built on the default stream, by
    whatever operator, may then be alive (the backward pass refuses leaves of its own inputs that are held so)."""
    xs, w_k, aux, _, offsets, slot, inv = RouteSort.apply(x, eps, w_in.shape[0], K, alpha)
    y = ExpertFFN.apply(xs, w_in, w_out, b_in, b_out, offsets, act)
    return Unsort.apply(y, w_k, residual, offsets, slot, inv), aux
