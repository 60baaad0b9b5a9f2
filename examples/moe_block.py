"""A stack of MoE blocks  h' = h + R_t * w_post * N(MoE(N(h) * w_pre)),  decoded token by token and trained for a step.

* ``decode``: a few tokens at a time -- the whole expert layer in ``moe_few``, the norms before and after it in one
  ``block_norm`` each (the norm after a block and the norm before the next are the same call).
* ``forward``: many tokens -- router, dispatch and expert FFN of the C ABI; ``block_norm`` takes the experts' rows straight
  out of the slot buffer, so that the gate-weighted combine costs no pass of its own.
* ``train_step``: gradients of one block with the activations of the norms kept in 8 bits (``BlockNorm``); the experts are
  plain torch products here, and the router's choices and scores are taken as they are.

    python examples/moe_block.py        # on a B200: both forms of the stack against each other, then training steps
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2401_13920_b200 import binding as B  # noqa: E402
from paper_2401_13920_b200 import block  # noqa: E402

EPS = 1e-6


@dataclass
class Layer:
    w_in: torch.Tensor      # [E][F][H] bf16
    w_out: torch.Tensor     # [E][H][F] bf16
    w_pre: torch.Tensor     # [H] fp32
    w_post: torch.Tensor    # [H] fp32


def make_layers(n, H, F, E, seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    r = lambda *s, std, mean=0.0, dt=torch.float32: (torch.randn(*s, generator=g, device=device) * std + mean).to(dt)
    bf = torch.bfloat16
    return [Layer(r(E, F, H, std=0.05, dt=bf), r(E, H, F, std=0.05, dt=bf), r(H, std=0.1, mean=1.0), r(H, std=0.1, mean=0.5)) for _ in range(n)]


def decode(layers, h):
    """The stack for a few tokens h [T][H] bf16: 2 launches a layer and 1 for the norms around it."""
    n = block.block_norm(h, w_pre=layers[0].w_pre, eps=EPS, want_h=False)[1]
    for i, l in enumerate(layers):
        y, _, w = block.moe_few(n, l.w_in, l.w_out, weighted=False)      # the score is applied after the norm
        last = i + 1 == len(layers)
        h, n, _ = block.block_norm(h, y, gate_w=w[0], w_post=l.w_post, w_pre=None if last else layers[i + 1].w_pre, eps=EPS, want_n=not last)
    return h


def forward(layers, h, capacity_factor=1.25):
    """The stack for many tokens, through the router and the dispatch buffer (tokens beyond the capacity keep their h)."""
    T, H = h.shape
    E, F = layers[0].w_in.shape[:2]
    shape = B.make_shape(T, H, E, 1, 1, h.dtype, B.LAYOUT_RECV)
    rule = B.CapacityRule(0.0, capacity_factor, -1.0, B.BOUND_BETA, 0)
    C = B.conventional_capacity(T, 1, E, capacity_factor)
    st = B.make_router(shape, C, rule, h.device)
    src = torch.zeros(T, dtype=torch.int32, device=h.device)
    h1 = torch.empty(st.rows, F, dtype=torch.bfloat16, device=h.device)
    y = torch.empty_like(st.buf)
    n = block.block_norm(h, w_pre=layers[0].w_pre, eps=EPS, want_h=False)[1]
    for i, l in enumerate(layers):
        B.locmoe_gate_route(shape, n, None, src, rule, st)
        B.locmoe_dispatch(shape, C, n, st.inv, st.buf, True, slot=st.slot)
        B.locmoe_expert_ffn(shape, C, F, st.buf, l.w_in, l.w_out, h1, y)
        last = i + 1 == len(layers)
        h, n, _ = block.block_norm(h, y, slot=st.slot, gate_w=st.gate_w, w_post=l.w_post, w_pre=None if last else layers[i + 1].w_pre,
                                   eps=EPS, want_n=not last)
    return h


def route(n, E, capacity_factor=1.25):
    """Router and placement of n [T][H]: a RouterState."""
    T, H = n.shape
    shape = B.make_shape(T, H, E, 1, 1, n.dtype, B.LAYOUT_RECV)
    rule = B.CapacityRule(0.0, capacity_factor, -1.0, B.BOUND_BETA, 0)
    st = B.make_router(shape, B.conventional_capacity(T, 1, E, capacity_factor), rule, n.device, with_buffer=False)
    B.locmoe_gate_route(shape, n, None, torch.zeros(T, dtype=torch.int32, device=n.device), rule, st)
    return st


def train_step(h, w_pre, w_in, w_out, w_post, w_next, target, checkpoint=True):
    """Loss and gradients of one block and the norm after it: ``loss = mean((n' - target)^2)``.  All weights require grad."""
    norm = dict(res_scale=1.0, eps=EPS, checkpoint=checkpoint, want_h=False)      # of h' nothing but its norm is used here
    _, n = block.BlockNorm.apply(h, None, None, None, w_pre, None, None, *norm.values())
    with torch.no_grad():
        st = route(n.detach(), w_in.shape[0])
    E, rows = w_in.shape[0], st.rows
    x = torch.where((st.inv >= 0)[:, None], n[st.inv.clamp_min(0).long()], 0.0).reshape(E, rows // E, -1)
    y = torch.bmm(torch.nn.functional.gelu(torch.bmm(x, w_in.transpose(1, 2))), w_out.transpose(1, 2)).reshape(rows, -1)
    _, n2 = block.BlockNorm.apply(h, y, st.gate_w, w_post, w_next, st.slot, st.inv, *norm.values())
    loss = (n2.float() - target).square().mean()
    loss.backward()
    return loss.detach()


def main():
    H, F, E = 2560, 10240, 32
    layers = make_layers(2, H, F, E)
    h = torch.randn(8, H, device="cuda").to(torch.bfloat16)
    a, b = decode(layers, h), forward(layers, h, capacity_factor=float(E))
    print("8 tokens, 2 layers: decode against the dispatched path: max difference %.3g of rms %.3g"
          % (float((a.float() - b.float()).abs().max()), float(b.float().square().mean().sqrt())))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for name, run in (("decode", lambda: decode(layers, h)), ("dispatched path", lambda: forward(layers, h, float(E)))):
        run()
        start.record()
        for _ in range(10):
            run()
        end.record()
        torch.cuda.synchronize()
        print("  %s: %.0f us a step" % (name, start.elapsed_time(end) * 100))
    T, H, F, E = 4096, 512, 1024, 8
    l = make_layers(1, H, F, E, seed=1)[0]
    h = torch.randn(T, H, device="cuda").to(torch.bfloat16)
    target = torch.randn(T, H, device="cuda")
    params = [l.w_pre, l.w_in, l.w_out, l.w_post, torch.ones(H, device="cuda")]
    params = [p.clone().requires_grad_() for p in params]
    for step in range(5):
        loss = train_step(h, *params, target)
        with torch.no_grad():
            for p in params:
                p -= 0.5 * p.grad.to(p.dtype)
                p.grad = None
        print("  training step %d with 8-bit checkpoints: loss %.5f" % (step, float(loss)))


if __name__ == "__main__":
    main()
