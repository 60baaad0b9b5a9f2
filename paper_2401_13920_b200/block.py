"""One MoE block around the router: the norms before and after it fused with its gate and residual, their gradient with
activations kept in 8 bits, and the whole expert layer for a few tokens.

The functions here allocate their outputs (and the workspace, from torch's allocator on the current stream) and call the
entry points of ``binding``; all arithmetic runs in the CUDA library.  With ``stream`` (a torch stream or a raw handle) the
whole call, its allocations among them, is made under that stream, as by ``with torch.cuda.stream(stream)``: the inputs have
to be ready there, and the outputs belong to it.  ``BlockNorm`` is the differentiable form.
"""
from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

try:   # 0.7 us a tensor; torch.empty takes 2.3, as much as a launch
    from torch._C._dynamo.guards import _empty_strided_cuda
except ImportError:   # no public name: a torch may have moved it
    def _empty_strided_cuda(size, stride, dtype):
        return torch.empty_strided(size, stride, dtype=dtype, device="cuda")


def _rows(n: int, width: int, dtype: torch.dtype) -> torch.Tensor:
    return _empty_strided_cuda((n, width), (width, 1), dtype)


def _flat(n: int, dtype: torch.dtype) -> torch.Tensor:
    return _empty_strided_cuda((n,), (1,), dtype)


_F32 = torch.float32


def _here(t: torch.Tensor, name: str) -> None:
    """Outputs, workspace and launch belong to the current device, so must the inputs.  The binding compares each tensor of a
    launch with it; here are those of calls that launch nothing (no rows), and host memory, before anything is allocated."""
    if not t.is_cuda or (t.numel() == 0 and t.get_device() != torch.cuda.current_device()):
        raise ValueError("%s: on %s, which is not the current CUDA device" % (name, t.device))


def _under(stream):
    """Context of a call on `stream`.  Its memory has to come from that stream's pool: the workspace goes back to its pool
    when the call returns, and only work of the same stream waits for the kernels that still use it."""
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        stream = torch.cuda.default_stream() if handle in (0, 1) else torch.cuda.ExternalStream(handle)   # 1: the legacy default
    return torch.cuda.stream(stream)


class Checkpoint(NamedTuple):
    """What the gradient needs of the forward pass, in 8 bits: the normalised rows (E4M3) and their reciprocal norms.
    ``u8`` / ``r_post`` are None where the block has no branch, ``x8`` / ``r_pre`` where it has no next norm."""
    u8: Optional[torch.Tensor]
    x8: Optional[torch.Tensor]
    r_post: Optional[torch.Tensor]
    r_pre: Optional[torch.Tensor]


def _count(*n: int) -> None:
    if max(n) > 2 ** 31 - 1:   # the library's counts have 32 bits, and ctypes cuts longer ones off without a word
        raise ValueError("a size of %d is too large" % max(n))


# Shape structs are read by a call and never written: one for each shape met, and the workspace sizes that go with them.
@lru_cache(maxsize=1024)
def _shape(T: int, H: int, E: int, dtype: torch.dtype) -> B.Shape:
    _count(T, H, E)
    return B.Shape(T, H, E, 1, 1, B.dtype_code(dtype), B.LAYOUT_SEND)


@lru_cache(maxsize=1024)
def _few_plan(T: int, H: int, E: int, K: int, F: int, dtype: torch.dtype):
    _count(K, F)
    shape = _shape(T, H, E, dtype)
    return shape, B.locmoe_moe_few_bytes(shape, K, F)


@lru_cache(maxsize=1024)
def _grad_bytes(T: int, H: int, dtype: torch.dtype, device: int) -> int:
    return B.locmoe_block_norm_grad_bytes(_shape(T, H, 1, dtype))


def _row_shape(like: torch.Tensor) -> tuple:
    """Shape struct, T and H for [T][H] tensors like this one."""
    if like.dim() != 2:
        raise ValueError("expected a [T][H] tensor, got %s" % (tuple(like.shape),))
    T, H = like.shape
    shape = _shape(T, H, 1, like.dtype)
    _here(like, "rows")
    return shape, T, H


def _want_rows(t, rows: int, H: int, name: str) -> None:
    """`t` (None: absent) is `rows` rows of H elements; how its other dimensions group them does not matter."""
    if t is not None and t.shape != (rows, H) and (t.shape[-1:] != (H,) or t.numel() != rows * H):
        raise ValueError("%s: expected %d rows of %d, got %s" % (name, rows, H, tuple(t.shape)))


def moe_few(x, w_in, w_out, K=1, eps=None, weighted=True, stream=None):
    """The whole MoE layer for a few tokens: x [T][H], w_in [E][F][H], w_out [E][H][F], all bf16, T <= 128.

    Returns ``(out, idx, w)``: out [T][H], the K chosen experts and their scores, [K][T] each."""
    if stream is not None:
        with _under(stream):
            return moe_few(x, w_in, w_out, K, eps, weighted)
    if x.dim() != 2 or w_in.dim() != 3 or w_out.dim() != 3:
        raise ValueError("expected x [T][H], w_in [E][F][H], w_out [E][H][F]")
    (T, H), (E, F, _) = x.shape, w_in.shape
    if w_in.shape[2] != H or w_out.shape != (E, H, F):
        raise ValueError("x %s, w_in %s and w_out %s do not belong together" % (tuple(x.shape), tuple(w_in.shape), tuple(w_out.shape)))
    _here(x, "x")
    if T > 0:
        shape, n = _few_plan(T, H, E, K, F, x.dtype)
    out, idx, w = _rows(T, H, x.dtype), _rows(K, T, torch.int32), _rows(K, T, _F32)
    if T == 0:
        return out, idx, w
    ws = _flat(n, torch.uint8)
    B.locmoe_moe_few(shape, x, K, F, w_in, w_out, idx, w, out, ws, eps, not weighted)
    return out, idx, w


def block_norm(h, y=None, slot=None, gate_w=None, w_post=None, w_pre=None, res_scale=1.0, eps=1e-6, checkpoint=False,
               want_h=True, want_n=True, stream=None):
    """h' = res_scale * h + gate_w * w_post * N(y[slot]),  n = w_pre * N(h').

    ``h`` is [T][H]; ``y`` the T tokens' rows (any beyond them are not read) or, with ``slot``, all rows of the slot buffer,
    also as [E][C][H] or [D][E][C][H].
    Returns ``(h_out, n, ckpt)``; ``h_out`` / ``n`` are None when not wanted, ``ckpt`` a ``Checkpoint`` or None.  Without
    ``y`` the block has no branch (the norm before the first block; ``want_h`` = False leaves out the copy of h)."""
    if stream is not None:
        with _under(stream):
            return block_norm(h, y, slot, gate_w, w_post, w_pre, res_scale, eps, checkpoint, want_h, want_n)
    if slot is not None and y is None:
        raise ValueError("y: needed with slot")
    shape, T, H = _row_shape(h)
    rows = T
    if y is not None and (slot is not None or y.shape != h.shape):
        have = y.numel() // max(H, 1)
        if slot is not None:
            rows = have
            _count(rows)
        _want_rows(y, max(have, rows), H, "y")
    h_out = _rows(T, H, h.dtype) if want_h else None
    n = _rows(T, H, h.dtype) if want_n else None
    u8 = x8 = r_post = r_pre = None
    if checkpoint and y is not None:
        u8, r_post = _rows(T, H, torch.float8_e4m3fn), _flat(T, _F32)
    if checkpoint and want_n:
        x8, r_pre = _rows(T, H, torch.float8_e4m3fn), _flat(T, _F32)
    if T > 0:
        B.locmoe_block_norm(shape, rows, h, y, slot, gate_w, w_post, w_pre, res_scale, eps, h_out, n, u8, x8, r_post, r_pre)
    return h_out, n, Checkpoint(u8, x8, r_post, r_pre) if checkpoint else None


def block_norm_grad(dh_out, dn, h_out=None, y=None, checkpoint: Optional[Checkpoint] = None, slot=None, inv=None, gate_w=None,
                    w_post=None, w_pre=None, res_scale=1.0, eps=1e-6, want_dh=True, want_dy=True, want_dgate=True,
                    want_dw=True, stream=None):
    """Gradient of ``block_norm`` from the gradients of h' and n (one may be None).

    The activations are ``h_out`` and ``y`` or, in their place, ``checkpoint``.  Returns ``(dh, dy, dgate, dw_post, dw_pre)``,
    each None when not wanted or not there.  With slots, ``dy`` has ``inv``'s rows, those without a token zero.
    All arrays of rows have exactly the rows that belong to them: T, or ``inv``'s for ``y`` with slots."""
    if stream is not None:
        with _under(stream):
            return block_norm_grad(dh_out, dn, h_out, y, checkpoint, slot, inv, gate_w, w_post, w_pre, res_scale, eps, want_dh, want_dy,
                                   want_dgate, want_dw)
    like = dn if dn is not None else dh_out
    if like is None:
        raise ValueError("dh_out, dn: one of them is needed")
    ck = checkpoint
    branch = (ck.u8 if ck is not None else y) is not None
    if slot is not None and inv is None:
        raise ValueError("inv: needed with slot (it says how many rows y has and which of them are empty)")
    shape, T, H = _row_shape(like)
    rows = T
    if branch and slot is not None:
        rows = inv.numel()
        _count(rows)
    _want_rows(dh_out, T, H, "dh_out")
    if ck is None:
        _want_rows(y, rows, H, "y")
        if dn is not None:
            _want_rows(h_out, T, H, "h_out")
    else:
        _want_rows(ck.u8, T, H, "checkpoint.u8")
        _want_rows(ck.x8, T, H, "checkpoint.x8")
    dh = _rows(T, H, like.dtype) if want_dh else None
    dy = _rows(rows, H, like.dtype) if want_dy and branch else None
    dgate = _flat(T, _F32) if want_dgate and branch else None
    dw_post = _flat(H, _F32) if want_dw and branch else None
    dw_pre = _flat(H, _F32) if want_dw and dn is not None else None
    if T == 0:
        for t in (dy, dw_post, dw_pre):
            if t is not None:
                t.zero_()
        return dh, dy, dgate, dw_post, dw_pre
    if dh is dy is dgate is dw_post is dw_pre is None:   # nothing is asked for that is there
        return dh, dy, dgate, dw_post, dw_pre
    ws = None
    if dw_post is not None or dw_pre is not None:
        ws = _flat(_grad_bytes(T, H, like.dtype, torch.cuda.current_device()), torch.uint8)
    acts = dict(u8=ck.u8, r_post=ck.r_post, x8=ck.x8 if dn is not None else None, r_pre=ck.r_pre if dn is not None else None) \
        if ck is not None else dict(y=y, h_out=h_out if dn is not None else None)
    B.locmoe_block_norm_grad(shape, rows, dh_out, dn, slot=slot if branch else None, inv=inv if branch and slot is not None else None,
                             gate_w=gate_w, w_post=w_post, w_pre=w_pre, res_scale=res_scale, eps=eps, dh=dh, dy=dy, dgate=dgate,
                             dw_post=dw_post, dw_pre=dw_pre, ws=ws, **acts)
    return dh, dy, dgate, dw_post, dw_pre


class BlockNorm(torch.autograd.Function):
    """``BlockNorm.apply(h, y, gate_w, w_post, w_pre, slot, inv, res_scale, eps, checkpoint, want_h) -> (h_out, n)``,
    differentiable in its first five arguments, once: the gradient of a gradient is an error.  With ``checkpoint`` the
    activations kept for the gradient are the 8-bit ones.  Without ``want_h`` h_out is None (the norm before the first block,
    whose h goes on as it is) and is formed only where the gradient needs it."""

    @staticmethod
    def forward(ctx, h, y, gate_w, w_post, w_pre, slot=None, inv=None, res_scale=1.0, eps=1e-6, checkpoint=False, want_h=True):
        same = y is None and res_scale == 1.0   # h' is h
        h_out, n, ck = block_norm(h, y, slot, gate_w, w_post, w_pre, res_scale, eps, checkpoint, want_h or not (checkpoint or same))
        ctx.consts = (res_scale, eps, ck is not None)
        ctx.y_shape = None if y is None else y.shape
        ctx.save_for_backward(gate_w, w_post, w_pre, slot, inv, *(ck if ck is not None else (y, h if h_out is None else h_out, None, None)))
        ctx.set_materialize_grads(False)
        return h_out if want_h else None, n

    @staticmethod
    @once_differentiable   # the kernels leave no graph: without it the results would pass as constants
    def backward(ctx, dh_out, dn):
        gate_w, w_post, w_pre, slot, inv, *acts = ctx.saved_tensors
        res_scale, eps, packed = ctx.consts
        if dh_out is None and dn is None:
            return (None,) * 11
        need = ctx.needs_input_grad
        dense = lambda t: None if t is None else t.contiguous()
        kw = dict(checkpoint=Checkpoint(*acts)) if packed else dict(y=acts[0], h_out=acts[1])
        dh, dy, dgate, dw_post, dw_pre = block_norm_grad(
            dense(dh_out), dense(dn), slot=slot, inv=inv, gate_w=gate_w, w_post=w_post, w_pre=w_pre, res_scale=res_scale, eps=eps,
            want_dh=need[0], want_dy=need[1], want_dgate=need[2], want_dw=need[3] or need[4], **kw)
        if dy is not None:
            if dy.numel() != ctx.y_shape.numel():
                raise ValueError("inv: %d rows, where y is %s" % (dy.shape[0], tuple(ctx.y_shape)))
            dy = dy.view(ctx.y_shape)
        if need[4] and w_pre is not None and dw_pre is None:   # n was not used: its weight has no gradient
            dw_pre = torch.zeros_like(w_pre)
        return (dh, dy if need[1] else None, dgate if need[2] else None, dw_post if need[3] else None, dw_pre if need[4] else None,
                None, None, None, None, None, None)
