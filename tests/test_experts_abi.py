"""Refusals of the calls on sorted tokens and of the experts' products on them: every bad argument is found on the host (no GPU
needed: nothing is launched)."""
import ctypes as C

import pytest
import torch

from tests.test_block_calls import StandIn

P = 1 << 20   # an address that is never followed: aligned, not NULL
BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def B():
    from paper_2401_13920_b200 import binding
    return binding


def _shape(B, T=4, H=64, E=8, dt=None):
    return B.Shape(T, H, E, 1, 1, B.BF16 if dt is None else dt, 0)


def test_struct_layouts_match_the_header(B):
    assert C.sizeof(B.SortGrad) == 9 * 8
    assert C.sizeof(B.ExpertLinear) == 7 * 8 + 8
    assert C.sizeof(B.ExpertLinearGrad) == 8 * 8 + 8


SORT = dict(idx=P, x=P, offsets=P, slot=P, inv=P, load=P, xs=P)


def _sort(B, shape=None, K=2, **kw):
    return B._lib.locmoe_sort(C.byref(shape or _shape(B)), K, *{**SORT, **kw}.values(), None)


UNSORT = dict(y=P, slot=P, w=P, residual=P, out=P)


def _unsort(B, shape=None, K=2, **kw):
    return B._lib.locmoe_unsort(C.byref(shape or _shape(B)), K, *{**UNSORT, **kw}.values(), None)


UNSORT_GRAD = dict(dout=P, y=P, offsets=P, slot=P, w=P, dy=P, dw=P)


def _unsort_grad(B, shape=None, K=2, **kw):
    return B._lib.locmoe_unsort_grad(C.byref(shape or _shape(B)), K, *{**UNSORT_GRAD, **kw}.values(), None)


def _sort_grad(B, shape=None, K=2, ws=P, ws_bytes=1 << 30, **kw):
    g = B.SortGrad(**{**dict(dxs=P, slot=P, x=P, eps=P, idx_k=P, dw=P, dp=P, dx=P, deps=P), **kw})
    return B._lib.locmoe_sort_grad(C.byref(shape or _shape(B)), K, C.byref(g), ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_sort, _unsort, _unsort_grad, _sort_grad])
def test_sizes_of_the_calls_on_sorted_tokens(B, call):
    assert call(B, K=0) == call(B, K=9) == -2
    assert call(B, _shape(B, T=0)) == call(B, _shape(B, H=0)) == call(B, _shape(B, E=0)) == -2
    assert call(B, _shape(B, dt=7)) == -3
    assert call(B, _shape(B, H=2048, E=2048)) == -7
    assert call(B, _shape(B, T=2 ** 30), K=2) == -7                            # K * T beyond 32 bits


def test_refusals_of_the_calls_on_sorted_tokens(B):
    for name in ("idx", "offsets", "slot", "inv"):
        assert _sort(B, **{name: None}) == -1 and _sort(B, **{name: P + 2}) == -4
    assert _sort(B, x=None) == _sort(B, xs=None) == -1 and _sort(B, x=P + 1) == _sort(B, xs=P + 1) == _sort(B, load=P + 1) == -4
    assert _sort(B, _shape(B, dt=B.F32), x=P + 2) == -4
    for name in ("y", "slot", "out"):
        assert _unsort(B, **{name: None}) == -1 and _unsort(B, **{name: P + 1}) == -4
    assert _unsort(B, residual=P + 1) == _unsort(B, w=P + 2) == -4
    assert _unsort_grad(B, dout=None) == _unsort_grad(B, offsets=None) == _unsort_grad(B, slot=None) == -1
    assert _unsort_grad(B, dy=None, dw=None) == _unsort_grad(B, y=None) == -1
    for name in UNSORT_GRAD:
        assert _unsort_grad(B, **{name: P + 1}) == -4
    assert _sort_grad(B, slot=None) == _sort_grad(B, dx=None) == _sort_grad(B, idx_k=None) == -1
    assert _sort_grad(B, x=None) == -1                                         # what belongs to the router needs the tokens
    assert _sort_grad(B, x=None, eps=None, dw=None, dp=None, deps=None, dxs=None) == -1
    assert _sort_grad(B, _shape(B, H=60)) == -2                                # groups of H / E
    assert _sort_grad(B, _shape(B, H=52 * 1001, E=52)) == -7                   # 52052 elements, no whole number of 16 bytes
    assert _sort_grad(B, ws=None) == _sort_grad(B, ws=P + 16) == -5
    assert _sort_grad(B, ws_bytes=B.locmoe_sort_grad_bytes(_shape(B)) - 1) == -5
    for name in ("dxs", "slot", "x", "eps", "idx_k", "dw", "dp", "dx", "deps"):
        assert _sort_grad(B, **{name: P + 1}) == -4
    assert B._lib.locmoe_sort_grad(C.byref(_shape(B)), 1, None, P, 1 << 30, None) == -1
    assert B._lib.locmoe_sort_grad_bytes(C.byref(_shape(B)), None) == -1


def _linear(B, shape=None, N=16, ws=P, ws_bytes=1 << 30, **kw):
    l = B.ExpertLinear(**{**dict(x=P, w=P, offsets=P, bias=P, residual=P, y=P, z=P, act=B.ACT_GELU), **kw})
    return B._lib.locmoe_expert_linear(C.byref(shape or _shape(B)), N, C.byref(l), ws, ws_bytes, None)


def _linear_grad(B, shape=None, N=16, ws=P, ws_bytes=1 << 30, **kw):
    l = B.ExpertLinearGrad(**{**dict(dy=P, x=P, w=P, offsets=P, z=P, dx=P, dw=P, db=P, act=B.ACT_GELU, dw_dtype=B.BF16), **kw})
    return B._lib.locmoe_expert_linear_grad(C.byref(shape or _shape(B)), N, C.byref(l), ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_linear, _linear_grad])
def test_expert_linear_refusals(B, call):
    grad = call is _linear_grad
    assert call(B, N=0) == call(B, N=12) == call(B, _shape(B, H=60)) == call(B, _shape(B, T=0)) == -2
    assert call(B, _shape(B, dt=B.F32)) == -3 and call(B, act=4) == call(B, act=-1) == -3
    assert call(B, N=1 << 20) == call(B, _shape(B, H=1 << 20)) == call(B, _shape(B, E=1032)) == call(B, _shape(B, T=2 ** 31 - 65536)) == -7
    names = ("dy", "x", "w", "offsets") if grad else ("x", "w", "offsets", "y")
    for name in names:
        assert call(B, **{name: None}) == -1 and call(B, **{name: P + 2}) == -4
    for name in ("z", "dx", "dw", "db") if grad else ("bias", "residual", "z"):
        assert call(B, **{name: P + 8}) == -4
    n = B.locmoe_expert_linear_bytes(_shape(B), 16, grad)
    assert n > 0 and n % 256 == 0
    assert call(B, ws=None) == call(B, ws=P + 16) == call(B, ws_bytes=n - 1) == -5
    if grad:
        assert call(B, dx=None, dw=None, db=None) == -1 and call(B, dw_dtype=2) == -3
    assert B._lib.locmoe_expert_linear_bytes(C.byref(_shape(B)), 16, 0, None) == -1
    assert B._lib.locmoe_expert_linear(C.byref(_shape(B)), 16, None, P, 1 << 30, None) == -1


T, H, K, E, N = 4, 64, 2, 8, 16
CALLS = dict(
    sort=dict(idx_k=(K * T, I32), offsets=(E + 1, I32), slot=(K * T, I32), inv=(K * T, I32), load=(E, I32), x=(T * H, BF), xs=(K * T * H, BF)),
    sort_grad=dict(slot=(K * T, I32), dx=(T * H, BF), dxs=(K * T * H, BF), x=(T * H, BF), eps=(E, F32), idx_k=(K * T, I32), dw=(K * T, F32), dp=(E, F32),
                   deps=(E, F32), ws=(1 << 20, U8)),
    unsort=dict(y=(K * T * H, BF), slot=(K * T, I32), out=(T * H, BF), w_k=(K * T, F32), residual=(T * H, BF)),
    unsort_grad=dict(dout=(T * H, BF), offsets=(E + 1, I32), slot=(K * T, I32), y=(K * T * H, BF), w_k=(K * T, F32), dy=(K * T * H, BF), dw=(K * T, F32)),
    expert_linear=dict(x=(T * H, BF), w=(E * N * H, BF), offsets=(E + 1, I32), y=(T * N, BF), ws=(1 << 20, U8), bias=(E * N, F32), residual=(T * N, BF),
                       z=(T * N, BF)),
    expert_linear_grad=dict(dy=(T * N, BF), offsets=(E + 1, I32), x=(T * H, BF), w=(E * N * H, BF), z=(T * H, BF), dx=(T * H, BF), dw=(E * N * H, BF),
                            db=(E * N, F32), ws=(1 << 20, U8)))


@pytest.mark.parametrize("which,name", [(w, n) for w, d in CALLS.items() for n in d])
def test_every_tensor_is_checked_before_the_launch(B, monkeypatch, which, name):
    called = []

    class Lib:
        def __getattr__(self, f):
            return lambda *a: called.append(f) or 0
    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda s: None)

    def call(**over):
        args = {**{k: StandIn(*v) for k, v in CALLS[which].items()}, **over}
        n = K if "linear" not in which else N
        return getattr(B, "locmoe_" + which)(_shape(B, T, H, E), n, **args)
    call()
    numel, dtype = CALLS[which][name]
    bad = [StandIn(numel, dtype, index=1), StandIn(numel, dtype, index=-1), StandIn(numel, torch.float16)]
    for t in bad + ([StandIn(numel - 1, dtype)] if name != "ws" else []):
        with pytest.raises(ValueError):
            call(**{name: t})
    assert len(called) == 1


def test_python_forms_refuse_what_does_not_fit():
    from paper_2401_13920_b200 import experts as X
    x, idx, w = torch.zeros(4, 16), torch.zeros(2, 4, dtype=I32), torch.zeros(3, 8, 16)
    order = X.Order(torch.zeros(4, dtype=I32), idx, torch.zeros(8, dtype=I32))
    for call in (lambda: X.sort_rows(x, idx, 3),                                         # host memory
                 lambda: X.sort_rows(x[0], idx, 3), lambda: X.sort_rows(x, idx[:, :3], 3), lambda: X.sort_rows(x, idx[0], 3),
                 lambda: X.sort_rows_grad(None, order), lambda: X.sort_rows_grad(x, order), lambda: X.sort_rows_grad(None, order, x, dw=x),
                 lambda: X.sort_rows_grad(torch.zeros(8, 16), order, dp=torch.zeros(3)), lambda: X.sort_rows_grad(None, order, x[:3]),
                 lambda: X.sort_rows_grad(None, order, x, eps=torch.zeros(4)),
                 lambda: X.sort_rows_grad(None, order, x, idx, dw=torch.zeros(4, 2)),
                 lambda: X.unsort_rows(x, order), lambda: X.unsort_rows(torch.zeros(8, 16), order, residual=x[:2]),
                 lambda: X.unsort_rows(torch.zeros(8, 16), order, w_k=torch.zeros(8)),
                 lambda: X.unsort_rows_grad(x, order, want_dy=False), lambda: X.unsort_rows_grad(x[:3], order),
                 lambda: X.expert_linear(x, w[0], order.offsets), lambda: X.expert_linear(x[:, :8], w, order.offsets),
                 lambda: X.expert_linear(x, w, order.offsets[:3]), lambda: X.expert_linear(x, w, order.offsets, act="tanh"),
                 lambda: X.expert_linear(x, w, order.offsets, bias=torch.zeros(8)),
                 lambda: X.expert_linear(x, w, order.offsets, residual=x),
                 lambda: X.expert_linear_grad(x[:, :8], x, w, order.offsets, want_dx=False, want_dw=False),
                 lambda: X.expert_linear_grad(x[:, :8], None, w, order.offsets),
                 lambda: X.expert_linear_grad(x[:, :8], x, w, order.offsets, z=x),
                 lambda: X.expert_linear_grad(x, x, w, order.offsets),
                 lambda: X.moe_layer(x, w, w, K=4)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: X.sort_rows(x.half(), idx, 3), lambda: X.unsort_rows_grad(x, order, y=torch.zeros(8, 16, dtype=BF)),
                 lambda: X.sort_rows_grad(torch.zeros(8, 16, dtype=BF), order, x),
                 lambda: X.expert_linear_grad(x[:, :8], x, w, order.offsets, dw_dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()
