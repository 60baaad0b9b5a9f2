"""Calls of the sorted-token operators and the layer made of them at the edges of what their documentation allows: no tokens, host
threads, captures, default types, and that nothing but the outputs is written."""
import ctypes as C
import os
import subprocess
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2401_13920_b200 import experts
    return experts


@pytest.fixture(scope="module")
def B():
    from paper_2401_13920_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("K", [1, 2])
def test_the_balance_loss_of_no_tokens(X, K):
    """Every output of the router may be the only one that a loss uses, also where there are no tokens."""
    for use in (0, 1, 2):
        x = torch.zeros(0, 64, dtype=BF, device="cuda", requires_grad=True)
        eps = torch.zeros(4, device="cuda", requires_grad=True)
        out = X.RouteSort.apply(x, eps, 4, K, 0.1)
        out[use].float().sum().backward()
        assert x.grad.shape == (0, 64) and x.grad.dtype == BF
        assert use == 0 and eps.grad is None or eps.grad.tolist() == [0.0] * 4


def test_the_weights_gradient_has_the_weights_type(X):
    g = gen(1)
    offsets = torch.tensor([0, 3, 3, 7], dtype=I32, device="cuda")
    x, dy, w = randn(g, 7, 16, dtype=BF), randn(g, 7, 24, dtype=BF), randn(g, 3, 24, 16)
    for rows in (7, 0):
        o = offsets if rows else torch.zeros_like(offsets)
        for wt in (F32, BF):
            _, dw, _ = X.expert_linear_grad(dy[:rows], x[:rows], w.to(wt), o, want_dx=False)
            _, same, _ = X.expert_linear_grad(dy[:rows], x[:rows], w.to(BF), o, want_dx=False, dw_dtype=wt)
            assert dw.dtype == wt and torch.equal(dw, same)


def at_once(calls, n=4000):
    """Straight calls of the library from a host thread each, which leave the interpreter's lock: {key: the codes they returned}."""
    codes = {k: set() for k in calls}

    def loop(k):
        f, args = calls[k]
        for _ in range(n):
            codes[k].add(f(*args))
    threads = [threading.Thread(target=loop, args=(k,)) for k in calls]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return codes


# What one thread asks of a kernel must not be taken away, between its check and its launch, by the smaller request of another.

def test_host_threads_order_by_different_numbers_of_experts(X, B):
    T, calls, kept = 64, {}, {}
    for E in (400, 600, 800, 1024):
        s = torch.cuda.Stream()
        idx = torch.randint(0, E, (1, T), generator=gen(E), device="cuda", dtype=I32)
        out = [torch.full((m,), -7, dtype=I32, device="cuda") for m in (E + 1, T, T)]
        shape = B.Shape(T, 1024, E, 1, 1, B.BF16, 0)
        kept[E] = (shape, idx, out, s)
        calls[E] = B._lib.locmoe_sort, (C.byref(shape), 1, idx.data_ptr(), None, *(t.data_ptr() for t in out), None, None, s.cuda_stream)
    codes = at_once(calls)
    assert all(c == {0} for c in codes.values()), codes
    for E, (_, idx, (offsets, slot, inv), _) in kept.items():
        order = torch.sort(idx[0], stable=True).indices
        assert torch.equal(inv, order.to(I32)) and torch.equal(slot[order.long()], torch.arange(T, device="cuda", dtype=I32))
        assert torch.equal(offsets[1:].long(), torch.bincount(idx[0].long(), minlength=E).cumsum(0))


def test_host_threads_run_the_router_on_rows_of_different_lengths(B):
    T, calls, kept = 32, {}, {}
    for H, E in ((16384, 512), (8192, 512), (4096, 128), (1024, 8)):
        s, x = torch.cuda.Stream(), randn(gen(H), T, H, dtype=BF)
        out = [torch.empty(T, dtype=t, device="cuda") for t in (I32, F32, F32)]
        shape, opts = B.Shape(T, H, E, 1, 1, B.BF16, 0), B.GateOpts(None, None, None, None, 0)
        B.locmoe_gate_ex(shape, x, *out)
        kept[H] = (shape, opts, s, x, out, [t.clone() for t in out])
        calls[H] = B._lib.locmoe_gate_ex, (C.byref(shape), x.data_ptr(), C.byref(opts), *(t.data_ptr() for t in out), s.cuda_stream)
    codes = at_once(calls)
    assert all(c == {0} for c in codes.values()), codes
    for *_, out, want in kept.values():
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_host_threads_run_the_norms_on_rows_of_different_lengths(B):
    T, calls, kept = 64, {}, {}
    for H in (512, 1024, 2048, 4096):
        s, h, dn = torch.cuda.Stream(), randn(gen(H), T, H), randn(gen(H + 1), T, H)
        n, dh, w = torch.empty_like(h), torch.empty_like(h), torch.ones(H, device="cuda")
        shape = B.Shape(T, H, 1, 1, 1, B.F32, 0)
        f = B.BlockNorm(h=h.data_ptr(), w_pre=w.data_ptr(), n_out=n.data_ptr(), res_scale=1.0, eps=1e-6)
        kept[H] = (shape, s, h, dn, n, dh, w, f)
        calls[H] = B._lib.locmoe_block_norm, (C.byref(shape), T, C.byref(f), s.cuda_stream)
    codes = at_once(calls)
    assert all(c == {0} for c in codes.values()), codes
    for _, _, h, _, n, *_ in kept.values():
        want = h.double() * (h.double().square().mean(1, keepdim=True) + 1e-6).rsqrt()
        # the sum of the squares, its root and the products: some steps of fp32
        assert ((n.double() - want).abs() <= (h.shape[1] + 8) * 2.0 ** -24 * want.abs()).all()


CHILD = """
import torch
from paper_2401_13920_b200 import experts
BF = torch.bfloat16
t = dict(x=torch.randn(40, 64, device="cuda").to(BF), w_in=torch.randn(4, 72, 64, device="cuda").to(BF), w_out=torch.randn(4, 64, 72, device="cuda").to(BF),
         residual=torch.randn(40, 64, device="cuda").to(BF))
leaf = t[LEAF].requires_grad_()
side = torch.cuda.Stream()
side.wait_stream(torch.cuda.current_stream())
def run():
    return experts.moe_layer(t["x"], t["w_in"], t["w_out"], 2, residual=t["residual"])[0].float().square().sum()
def under(stream, f):
    with torch.cuda.stream(stream):
        return f()
def capture():
    leaf.grad = None
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph):
            run().backward()
        graph.replay()
        torch.cuda.synchronize()
        got, leaf.grad = leaf.grad, None
        assert torch.equal(got, torch.autograd.grad(run(), leaf)[0])
        print("captured")
    except RuntimeError as e:
        print("refused" if "a captured backward pass" in str(e) else e)
    torch.cuda.synchronize()
default = torch.cuda.default_stream()
under(side, lambda: run().backward())                   # a pass before any capture
torch.cuda.synchronize()
other, layer = (default, side) if FIRST == "default" else (side, default)
kept = under(other, lambda: leaf * 1.0)                 # the leaf's node belongs to another operator's stream ...
graph = under(layer, run)                               # ... and the layer sees it on one that says otherwise
torch.cuda.synchronize()
capture()
del kept, graph
capture()
"""


@pytest.mark.parametrize("leaf", ["x", "w_in", "w_out", "residual"])
@pytest.mark.parametrize("first,want", [("default", "refused"), ("side", "captured")])
def test_a_captured_backward_pass_knows_where_a_leafs_node_was_made(leaf, first, want):
    """In a process of its own, which has to live on."""
    code = CHILD.replace("LEAF", repr(leaf)).replace("FIRST", repr(first))
    done = subprocess.run([sys.executable, "-W", "ignore", "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    assert done.stdout.split() == [want, "captured"], done.stdout


def test_asking_for_a_leafs_stream_leaves_the_leaf_alone(X):
    """Its own hooks are for gradients: not called, and kept in their order; no gradient appears."""
    calls = []
    x = torch.ones(4, device="cuda", requires_grad=True)
    for f in (3.0, 5.0):
        x.register_hook(lambda g, f=f: calls.append(f) or g + f * len(calls))
    side = torch.cuda.Stream()
    for stream, handle in ((torch.cuda.default_stream(), 0), (side, side.cuda_stream)):
        with torch.cuda.stream(stream):
            kept = x * 2.0
        assert X._leaf_stream(x) == handle and not calls and x.grad is None
        del kept
    (x * 2.0).sum().backward()
    assert calls == [3.0, 5.0] and x.grad.tolist() == [2.0 + 3.0 + 10.0] * 4


MARGIN = 4096


class Guarded:
    """Arrays in the middle of buffers of a fixed pattern: outputs, whose margins have to stay, and inputs, which have to stay."""

    def __init__(self):
        self.kept = []

    def _place(self, n):
        buf = torch.empty(n + 2 * MARGIN, dtype=U8, device="cuda")
        buf.copy_((torch.arange(buf.numel(), device="cuda") * 37 + 11).to(U8))
        return buf

    def output(self, dtype, *shape):
        n = torch.empty(0, dtype=dtype).element_size()
        for s in shape:
            n *= s
        buf = self._place(n)
        self.kept.append((buf, buf.clone(), n))
        return buf[MARGIN:MARGIN + n].view(dtype).view(shape)

    def input(self, t):
        n = t.numel() * t.element_size()
        buf = self._place(n)
        inner = buf[MARGIN:MARGIN + n].view(t.dtype).view(t.shape)
        inner.copy_(t)
        self.kept.append((buf, buf.clone(), 0))
        return inner

    def check(self):
        torch.cuda.synchronize()
        for buf, was, n in self.kept:
            at = MARGIN if n else buf.numel()
            assert torch.equal(buf[:at], was[:at]) and torch.equal(buf[at + n:], was[at + n:])


OFFSETS = [[0, 1, 2, 3, 4], [0, 0, 5, 6, 7], [1, 2, 2, 5, 6], [0, 90, 20, 2 ** 31 - 1, 70], [-5, -2 ** 31, 30, 10, 500], [70, 70, 0, 0, -1], [2 ** 31 - 1] * 5,
           [0, 40, 40, 41, 66], [7, 0, 7, 0, 7], [0, 2 ** 31 - 1, 0, 2 ** 31 - 1, 0]]


@pytest.mark.parametrize("offsets", OFFSETS)
@pytest.mark.parametrize("R", [1, 7, 70, 131])
def test_products_write_their_outputs_and_nothing_else(X, B, R, offsets):
    """Ordinary offsets, and such as descend or leave the rows, in the form without tiles, with them, and every gradient."""
    g, E, IN, OUT = gen(R), 4, 72, 264
    G = Guarded()
    o = G.input(torch.tensor(offsets, dtype=I32, device="cuda"))
    x, w, dy, z = (G.input(t) for t in (randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF), randn(g, R, OUT, dtype=BF), randn(g, R, IN, dtype=BF)))
    bias, res = G.input(randn(g, E, OUT)), G.input(randn(g, R, OUT, dtype=BF))
    shape = B.Shape(R, IN, E, 1, 1, B.BF16, 0)
    ws = G.output(U8, B.locmoe_expert_linear_bytes(shape, OUT))
    B.locmoe_expert_linear(shape, OUT, x, w, o, G.output(BF, R, OUT), ws, bias, res, G.output(BF, R, OUT), B.ACT_GELU)
    ws = G.output(U8, B.locmoe_expert_linear_bytes(shape, OUT, True))
    for dwt in (BF, F32):
        B.locmoe_expert_linear_grad(shape, OUT, dy, o, x, w, z, G.output(BF, R, IN), G.output(dwt, E, OUT, IN), G.output(F32, E, OUT), B.ACT_SILU, ws)
    B.locmoe_expert_linear_grad(shape, OUT, dy, o, db=G.output(F32, E, OUT))
    G.check()
    assert B.locmoe_device_flags() == 0


def test_split_products_write_their_outputs_and_nothing_else(X, B):
    """Few tiles with a long reduction, in runs that leave sums in the workspace."""
    g, E, R, IN, OUT = gen(3), 2, 1200, 2048, 136
    for offsets in ([0, 1100, 1190], [3, 2 ** 31 - 1, 40]):
        G = Guarded()
        o = G.input(torch.tensor(offsets, dtype=I32, device="cuda"))
        x, w, dy = (G.input(t) for t in (randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF), randn(g, R, OUT, dtype=BF)))
        shape = B.Shape(R, IN, E, 1, 1, B.BF16, 0)
        B.locmoe_expert_linear(shape, OUT, x, w, o, G.output(BF, R, OUT), G.output(U8, B.locmoe_expert_linear_bytes(shape, OUT)))
        B.locmoe_expert_linear_grad(shape, OUT, dy, o, x, w, None, G.output(BF, R, IN), G.output(F32, E, OUT, IN), G.output(F32, E, OUT), B.ACT_NONE,
                                    G.output(U8, B.locmoe_expert_linear_bytes(shape, OUT, True)))
        G.check()
    assert B.locmoe_device_flags() == 0


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,K,H,E", [(5, 2, 72, 4), (33, 3, 777, 7), (1500, 2, 96, 8), (700, 5, 40, 5)])
def test_rows_are_written_and_nothing_else(X, B, T, K, H, E, dt):
    """Choices that are no experts, slots that are no rows, offsets that promise more or fewer rows than there are."""
    g, G = gen(T), Guarded()
    V, code = K * T, B.F32 if dt is F32 else B.BF16
    shape = B.Shape(T, H, E, 1, 1, code, 0)
    wild = torch.tensor([-1, -7, E, 2 ** 31 - 1, -2 ** 31], dtype=I32, device="cuda")
    idx = torch.randint(0, E, (K, T), generator=g, device="cuda", dtype=I32)
    idx = G.input(torch.where(torch.rand(K, T, generator=g, device="cuda") < 0.3, wild[torch.randint(0, 5, (K, T), generator=g, device="cuda")], idx))
    x, y, dout = G.input(randn(g, T, H, dtype=dt)), G.input(randn(g, V, H, dtype=dt)), G.input(randn(g, T, H, dtype=dt))
    w, eps, dp = G.input(randn(g, K, T)), G.input(randn(g, E)), G.input(randn(g, E))
    offsets, slot, inv = G.output(I32, E + 1), G.output(I32, K, T), G.output(I32, V)
    B.locmoe_sort(shape, K, idx, offsets, slot, inv, G.output(I32, E), x, G.output(dt, V, H))
    B.locmoe_sort(shape, K, idx, offsets, slot, inv, None)
    bad = torch.where(torch.rand(K, T, generator=g, device="cuda") < 0.2, torch.tensor(2 ** 31 - 1, dtype=I32, device="cuda"), slot)
    bad = G.input(torch.where(torch.rand(K, T, generator=g, device="cuda") < 0.2, torch.tensor(V, dtype=I32, device="cuda"), bad))
    for s in (slot, bad):
        for last in (None, -5, V, 2 ** 31 - 1):
            o = offsets
            if last is not None:
                o = offsets.clone()
                o[E] = last
                o = G.input(o)
            B.locmoe_unsort_grad(shape, K, dout, o, s, y, w, G.output(dt, V, H), G.output(F32, K, T))
        B.locmoe_unsort(shape, K, y, s, G.output(dt, T, H), w, dout)
        if H % E == 0:
            B.locmoe_sort_grad(shape, K, s, G.output(dt, T, H), y, x, eps, idx, w, dp, G.output(F32, E), G.output(U8, B.locmoe_sort_grad_bytes(shape)))
        B.locmoe_sort_grad(shape, K, s, G.output(dt, T, H), y)
    G.check()
    assert B.locmoe_device_flags() == 0
