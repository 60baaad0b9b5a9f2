"""The blocks of the example: the few-token path against the dispatched one, and a training step against autograd in 64 bits."""
import math
import os
import sys

import pytest
import torch

from tests.test_block_norm_gpu import _forward64, _grad64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import moe_block
    finally:
        sys.path.pop(0)
    return moe_block


@pytest.mark.parametrize("T", [1, 6, 24, 100])
def test_decode_agrees_with_the_dispatched_stack(X, T):
    layers = X.make_layers(1, 512, 1024, 8, seed=3)
    h = torch.randn(T, 512, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").to(torch.bfloat16)
    a, b = X.decode(layers, h), X.forward(layers, h, capacity_factor=8.0)
    # both round y to bf16 (2^-8 of an element), the dispatched path also the GeLU's result (2^-8 of a row's norm spread over
    # its elements); the branch is R w_post N(y) with R < 1, w_post < 1.1, and h' is rounded to bf16 once on either side
    branch = 1.1 * (2 ** -8 * 6 / math.sqrt(3) + 2 ** -8 * 8)
    tol = branch + 2 * 2.0 ** -8 * b.float().abs()
    assert ((a.float() - b.float()).abs() <= tol).all()


class Packed64(torch.autograd.Function):
    """The block norm in 64 bits with the gradient that 8-bit checkpoints stand for: the formulas at the rounded rows."""

    @staticmethod
    def forward(ctx, h, y, gate_w, w_post, w_pre, slot, inv, eps):
        s = dict(h=h, y=y, slot=slot, inv=inv, gate_w=gate_w, w_post=w_post, w_pre=w_pre)
        hp, n, u, x, r, q = _forward64(s, 1.0, eps)
        code = lambda t: t.float().to(torch.float8_e4m3fn).double()
        ctx.s, ctx.act = {k: t if t is None else t.detach() for k, t in s.items()}, (code(u), code(x), r, q)
        return hp, n

    @staticmethod
    def backward(ctx, dh_out, dn):
        dh, dy, k, dwp, dwn, _ = _grad64(dict(ctx.s, dh_out=dh_out, dn=dn), 1.0, 0.0, ctx.act)
        branch = ctx.s["y"] is not None
        return dh, dy if branch else None, None, dwp if branch else None, dwn, None, None, None


def exact64(h, y, gate_w, w_post, w_pre, slot, inv, eps):
    norm = lambda v: v * (v.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    hp = h
    if y is not None:
        hp = h + gate_w[:, None] * w_post * norm(torch.where((slot >= 0)[:, None], y[slot.clamp_min(0).long()], 0.0))
    return hp, norm(hp) * w_pre


@pytest.mark.parametrize("checkpoint", [False, True])
def test_training_step(X, checkpoint):
    T, H, F, E = 192, 64, 128, 4
    l = X.make_layers(1, H, F, E, seed=5)[0]
    g = torch.Generator(device="cuda").manual_seed(7)
    h = torch.randn(T, H, generator=g, device="cuda")
    target = torch.randn(T, H, generator=g, device="cuda")
    p = [t.float().clone().requires_grad_() for t in (l.w_pre, l.w_in, l.w_out, l.w_post, torch.ones(H, device="cuda"))]
    hh = h.clone().requires_grad_()
    loss = X.train_step(hh, *p, target, checkpoint)
    # the same in 64 bits, with the router's choices, slots and scores taken as constants; torch's own differentiation
    # where the activations are kept, the formulas at the rounded rows where the checkpoints are
    block = Packed64.apply if checkpoint else exact64
    q = [t.detach().double().requires_grad_() for t in p]
    h64 = h.double().requires_grad_()
    n = block(h64, None, None, None, q[0], None, None, X.EPS)[1]
    st = X.route(X.block.block_norm(h, w_pre=p[0].detach(), eps=X.EPS, want_h=False)[1], E)
    x = torch.where((st.inv >= 0)[:, None], n[st.inv.clamp_min(0).long()], 0.0).reshape(E, st.rows // E, -1)
    y = torch.bmm(torch.nn.functional.gelu(torch.bmm(x, q[1].transpose(1, 2))), q[2].transpose(1, 2)).reshape(st.rows, -1)
    n2 = block(h64, y, st.gate_w.double(), q[3], q[4], st.slot, st.inv, X.EPS)[1]
    want = (n2 - target.double()).square().mean()
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 1e-5 * float(want.detach())
    for a, b in zip([hh] + p, [h64] + q):
        assert float((a.grad.double() - b.grad).norm()) <= 2e-5 * float(b.grad.norm()) + 1e-12
