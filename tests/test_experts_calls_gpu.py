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
