"""Refusals of the block's entry points: every bad argument is found on the host (no GPU needed: nothing is launched)."""
import ctypes as C

import pytest
import torch

P = 1 << 20   # an address that is never followed: aligned, not NULL


@pytest.fixture(scope="module")
def B():
    from paper_2401_13920_b200 import binding
    return binding


def _few(B, shape=None, x=P, K=1, F=64, w_in=P, w_out=P, flags=0, idx=P, w=P, out=P, ws=P, ws_bytes=1 << 30, eps=None):
    sh = shape if shape is not None else B.make_shape(4, 64, 8, 1, 1, B.BF16)
    return B._lib.locmoe_moe_few(C.byref(sh), x, eps, K, F, w_in, w_out, flags, idx, w, out, ws, ws_bytes, None)


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B.BlockNorm) == 12 * 8 + 8
    assert C.sizeof(B.BlockNormGrad) == 18 * 8 + 8


def test_moe_few_refusals(B):
    mk = lambda **k: B.make_shape(**{**dict(T=4, H=64, E=8, n_nodes=1, dev_per_node=1, x_dtype=B.BF16), **k})
    n = B.locmoe_moe_few_bytes(mk(), 1, 64)
    assert n > 0 and n % 256 == 0 and n <= B.locmoe_moe_few_bytes(mk(), 2, 64)
    for name in ("x", "w_in", "w_out", "idx", "w", "out"):
        assert _few(B, **{name: None}) == -1, name
    assert _few(B, mk(x_dtype=B.F32)) == -3                       # bf16 only
    assert _few(B, flags=2) == -3 and _few(B, flags=B.FEW_UNWEIGHTED, K=2) == -2
    assert _few(B, K=0) == _few(B, K=9) == -2 and _few(B, mk(E=4), K=5) == -2
    assert _few(B, F=0) == _few(B, F=12) == -2
    assert _few(B, mk(H=60, E=4)) == -2                           # H no multiple of 8
    assert _few(B, mk(T=129)) == -7 and _few(B, mk(T=0)) == -2
    assert _few(B, mk(H=2048 * 8, E=2048)) == -7 and _few(B, F=1 << 20) == -7
    for name in ("x", "w_in", "w_out", "out"):
        assert _few(B, **{name: P + 8}) == -4, name
    assert _few(B, idx=P + 2) == _few(B, w=P + 1) == _few(B, eps=P + 2) == -4
    assert _few(B, ws=None) == _few(B, ws=P + 16) == _few(B, ws_bytes=n - 1) == -5
    out = C.c_size_t()
    assert B._lib.locmoe_moe_few_bytes(C.byref(mk()), 1, 64, None) == -1
    assert B._lib.locmoe_moe_few_bytes(None, 1, 64, C.byref(out)) == -1
    assert B._lib.locmoe_moe_few_bytes(C.byref(mk(E=7)), 1, 64, C.byref(out)) == -2     # H % E


def _norm(B, shape=None, C_alloc=1, **kw):
    sh = shape if shape is not None else B.Shape(4, 64, 1, 1, 1, B.BF16, 0)
    b = B.BlockNorm(**{**dict(h=P, h_out=P, n_out=P, res_scale=1.0, eps=1e-6), **kw})
    return B._lib.locmoe_block_norm(C.byref(sh), C_alloc, C.byref(b), None)


def test_block_norm_refusals(B):
    assert B._lib.locmoe_block_norm(C.byref(B.Shape(4, 64, 1, 1, 1, B.BF16, 0)), 1, None, None) == -1
    assert _norm(B, h=None) == -1 and _norm(B, h_out=None, n_out=None) == -1
    assert _norm(B, slot=P) == -1 and _norm(B, u8=P, r_post=P) == -1            # no branch to take them from
    assert _norm(B, y=P, u8=P) == _norm(B, y=P, r_post=P) == _norm(B, x8=P) == _norm(B, r_pre=P) == -1   # pairs
    assert _norm(B, eps=-1.0) == _norm(B, eps=float("nan")) == _norm(B, res_scale=float("nan")) == -2
    assert _norm(B, B.Shape(4, 200008, 1, 1, 1, B.BF16, 0), x8=P, r_pre=P) == -2   # sqrt(H) beyond the codes' range
    assert _norm(B, C_alloc=0, y=P, slot=P) == -2                                 # rows of the slot buffer
    assert _norm(B, B.Shape(4, 64, 1, 1, 1, 7, 0)) == -3
    assert _norm(B, h=P + 1) == _norm(B, y=P + 1) == _norm(B, gate_w=P + 2) == _norm(B, w_pre=P + 1) == -4


def _grad(B, shape=None, C_alloc=1, ws=P, ws_bytes=1 << 40, **kw):
    sh = shape if shape is not None else B.Shape(4, 64, 1, 1, 1, B.BF16, 0)
    b = B.BlockNormGrad(**{**dict(dh_out=P, dn=P, h_out=P, y=P, dh=P, res_scale=1.0, eps=1e-6), **kw})
    return B._lib.locmoe_block_norm_grad(C.byref(sh), C_alloc, C.byref(b), ws, ws_bytes, None)


def test_block_norm_grad_refusals(B):
    sh = B.Shape(4, 64, 1, 1, 1, B.BF16, 0)
    n = B.locmoe_block_norm_grad_bytes(sh)
    assert n > 0 and n % 256 == 0
    assert B._lib.locmoe_block_norm_grad_bytes(C.byref(sh), None) == -1
    assert _grad(B, dh_out=None, dn=None) == -1 and _grad(B, h_out=None) == -1 and _grad(B, dh=None) == -1
    assert _grad(B, dw_pre=P, dn=None) == -1 and _grad(B, y=None, dy=P) == _grad(B, y=None, dgate=P) == _grad(B, y=None, slot=P) == -1
    assert _grad(B, inv=P) == -1                                                  # inv without slot
    assert _grad(B, x8=P, r_pre=P) == -3                                          # both forms of the activations
    assert _grad(B, h_out=None, y=None, x8=P) == _grad(B, h_out=None, y=None, x8=P, r_pre=P, u8=P) == -1
    assert _grad(B, eps=-1.0) == -2 and _grad(B, slot=P, C_alloc=0) == -2
    assert _grad(B, dw_post=P, ws=None) == _grad(B, dw_post=P, ws=P + 8) == _grad(B, dw_pre=P, ws_bytes=n - 1) == -5
    assert _grad(B, dh=P + 1) == _grad(B, dgate=P + 2) == -4


def test_python_forms_refuse_what_does_not_fit():
    from paper_2401_13920_b200 import block
    x, wi, wo = torch.zeros(2, 16), torch.zeros(4, 8, 16), torch.zeros(4, 16, 8)
    with pytest.raises(ValueError):
        block.moe_few(x[0], wi, wo)
    with pytest.raises(ValueError):
        block.moe_few(x, wi, wo.transpose(1, 2))
    with pytest.raises(ValueError):
        block.block_norm(torch.zeros(2, 16), torch.zeros(2, 8))
    with pytest.raises(ValueError):
        block.block_norm_grad(x, x, x, x, slot=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        block.block_norm(torch.zeros(2, 16, dtype=torch.float16))
    with pytest.raises(ValueError):                                               # host memory
        block.block_norm(torch.zeros(2, 16))
    with pytest.raises(ValueError):
        block.block_norm(torch.zeros(16, 2).t())
