"""The whole MoE layer for a few tokens on the GPU against a plain implementation in 64 bits.

Tolerances: the GeLU's result is rounded to bf16 (each term of the second product off by at most 2^-9 of itself, taken as
independent: six deviations of 2^-9 / sqrt 3 of the terms' root-sum-square), all sums are fp32 (1e-6 of the terms' absolute
sum), the output is rounded once to bf16 (2^-8 of the value bounds half a unit in the last place).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2401_13920_b200 import block
    return block


def _inputs(T, H, F, E, seed, bias=False, std=0.05):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std
    bf = torch.bfloat16
    return r(T, H).to(bf), r(E, F, H, std=std).to(bf), r(E, H, F, std=std).to(bf), r(E, std=0.05) if bias else None


def _reference(x, w_in, w_out, K, eps, weighted=True):
    T, H = x.shape
    E = w_in.shape[0]
    G = x.double().reshape(T, E, H // E).mean(2) + (eps.double() if eps is not None else 0.0)
    G = G.clamp_min(0.0)
    p = torch.softmax(G, 1)
    order = torch.sort(G, dim=1, descending=True, stable=True)
    idx = order.indices[:, :K]
    # distance to the nearest other order of the first K + 1 logits
    v = order.values[:, :K + 1]
    gap = torch.where(v[:, 1:] > 0, v[:, :-1] - v[:, 1:], 1.0).amin(1) if v.shape[1] > 1 else torch.ones(T, device="cuda", dtype=torch.float64)
    out = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    sq, ab = torch.zeros_like(out), torch.zeros_like(out)
    w = p.gather(1, idx)
    for c in range(K):
        for e in idx[:, c].unique().tolist():
            t = torch.nonzero(idx[:, c] == e).squeeze(1)
            a = x[t].double() @ w_in[e].double().t()
            a = 0.5 * a * torch.erfc(-a / math.sqrt(2.0))
            f = (w[t, c] if weighted else torch.ones_like(w[t, c]))[:, None]
            wo = w_out[e].double()
            out[t] += f * (a @ wo.t())
            sq[t] += f * f * (a.pow(2) @ wo.pow(2).t())
            ab[t] += f * (a.abs() @ wo.abs().t())
    return idx.t(), w.t(), gap, out, sq.sqrt(), ab


def _check(got, ref):
    (out, idx, w), (ri, rw, gap, ro, sq, ab) = got, ref
    clear = gap > 1e-6                      # choices may differ only within 1e-6 of a tie
    assert clear.float().mean() > 0.9
    assert torch.equal(idx[:, clear].long(), ri[:, clear])
    assert torch.allclose(w[:, clear].double(), rw[:, clear], rtol=2e-6)
    tol = 6 * 2.0 ** -9 / math.sqrt(3.0) * sq + 2.0 ** -8 * ro.abs() + 1e-6 * ab + 1e-9
    err = (out.double() - ro).abs()
    assert (err[clear] <= tol[clear]).all(), float((err / tol)[clear].max())


CASES = [(1, 64, 64, 1, 1), (1, 8, 8, 1, 1), (1, 1024, 4096, 8, 1), (2, 8, 16, 2, 2), (3, 520, 1032, 4, 1), (4, 96, 72, 12, 3), (8, 256, 512, 8, 1),
         (5, 1024, 1032, 16, 3), (9, 2560, 2568, 32, 1), (13, 1560, 808, 24, 3), (16, 320, 640, 32, 8), (17, 320, 640, 4, 1), (33, 256, 264, 8, 2),
         (64, 512, 1024, 16, 2), (100, 136, 200, 17, 5), (128, 1024, 256, 1024, 1), (128, 512, 512, 64, 8), (128, 64, 128, 2, 1), (128, 256, 512, 1, 1),
         (1, 256, 5120, 4, 1), (2, 64, 16384, 2, 1), (7, 40, 8, 5, 1)]


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("T,H,F,E,k", CASES)
def test_layer(K, T, H, F, E, k, bias):
    x, w_in, w_out, eps = _inputs(T, H, F, E, T + H + F, bias)
    _check(K.moe_few(x, w_in, w_out, K=k, eps=eps), _reference(x, w_in, w_out, k, eps))


@pytest.mark.parametrize("T,F,k", [(8, 4096, 1), (16, 512, 1), (16, 512, 2), (32, 520, 1), (70, 264, 1), (128, 512, 2)])
def test_all_tokens_on_one_expert(K, T, F, k):
    """Every token's first choice is the same expert: one, two or more chunks of tokens for one weight row."""
    x, w_in, w_out, _ = _inputs(T, 512, F, 8, T)
    eps = torch.zeros(8, device="cuda")
    eps[5] = 3.0
    got = K.moe_few(x, w_in, w_out, K=k, eps=eps)
    assert (got[1][0] == 5).all()
    _check(got, _reference(x, w_in, w_out, k, eps))


@pytest.mark.parametrize("T,F,k,one", [(17, 18952, 1, False), (17, 18952, 1, True), (40, 19000, 2, False), (128, 18944, 1, False), (128, 19000, 2, True)])
def test_wide_layer_with_many_tokens_an_expert(K, T, F, k, one):
    """The tiles of 32 tokens: one to four of them an expert, rows and k that end inside a tile."""
    x, w_in, w_out, eps = _inputs(T, 264, F, 4, F, bias=True)
    if one:
        eps = torch.tensor([0.0, 0.0, 3.0, 0.0], device="cuda")
    _check(K.moe_few(x, w_in, w_out, K=k, eps=eps), _reference(x, w_in, w_out, k, eps))


def test_ties_go_to_the_lower_index(K):
    """Logits that the ReLU made 0 are equal: their experts are chosen in index order, with equal scores."""
    x, w_in, w_out, _ = _inputs(3, 128, 64, 8, 1)
    x = -x.abs()
    out, idx, w = K.moe_few(x, w_in, w_out, K=4)
    assert idx.t().tolist() == [[0, 1, 2, 3]] * 3 and torch.allclose(w, torch.full_like(w, 1 / 8))


def test_unweighted(K):
    x, w_in, w_out, _ = _inputs(11, 256, 512, 8, 2)
    r = _reference(x, w_in, w_out, 1, None, weighted=False)
    _check(K.moe_few(x, w_in, w_out, weighted=False), r)


@pytest.mark.parametrize("T", [4, 12, 40])
def test_infinities_and_nan_stay_in_their_tokens(K, T):
    x, w_in, w_out, _ = _inputs(T, 256, 264, 8, 3)
    clean = K.moe_few(x, w_in, w_out, K=2)
    y = x.clone()
    y[0, 3], y[1, 200], y[2, 7] = float("nan"), float("inf"), float("-inf")
    y[2] = float("-inf")
    out, idx, w = K.moe_few(y, w_in, w_out, K=2)
    assert torch.equal(out[3:], clean[0][3:]) and torch.equal(idx[:, 3:], clean[1][:, 3:])
    assert (idx >= 0).all() and (idx < 8).all() and (idx[0] != idx[1]).all()


@pytest.mark.parametrize("T,k", [(1, 1), (8, 1), (12, 2), (50, 3)])
def test_bits_repeat_also_on_another_stream_and_in_a_graph(K, T, k):
    x, w_in, w_out, _ = _inputs(T, 1024, 4096, 8, 4)
    one = K.moe_few(x, w_in, w_out, K=k)
    for _ in range(3):
        two = K.moe_few(x, w_in, w_out, K=k)
        assert all(torch.equal(a, b) for a, b in zip(one, two))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        two = K.moe_few(x, w_in, w_out, K=k)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    graph = torch.cuda.CUDAGraph()
    xs = x.clone()
    with torch.cuda.graph(graph):
        three = K.moe_few(xs, w_in, w_out, K=k)
        four = K.moe_few(three[0], w_in, w_out, K=k)      # a second layer follows at once
    xs.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, three))
    assert torch.equal(four[0], K.moe_few(one[0], w_in, w_out, K=k)[0])


def test_agrees_with_the_dispatched_layer(K):
    """The same tokens through gate, capacity, route, dispatch, expert FFN and combine with room for all of them."""
    from paper_2401_13920_b200 import binding as B
    T, H, F, E = 40, 512, 1024, 8
    x, w_in, w_out, _ = _inputs(T, H, F, E, 5)
    sh = B.make_shape(T, H, E, 1, 2, torch.bfloat16, B.LAYOUT_RECV)
    rule = B.CapacityRule(0.0, float(2 * E), -1.0, B.BOUND_BETA, 0)
    st = B.make_router(sh, T, rule)
    src = (torch.arange(T, device="cuda") % 2).to(torch.int32)
    h1 = torch.empty(st.rows, F, dtype=torch.bfloat16, device="cuda")
    y, out = torch.empty_like(st.buf), torch.empty_like(x)
    B.locmoe_moe_layer(sh, x, src, None, rule, T, F, w_in, w_out, B.layer_buffers(st, h1, y), out)
    got = K.moe_few(x, w_in, w_out)
    assert (st.drop == 0).all() and torch.equal(got[1][0], st.idx)
    r = _reference(x, w_in, w_out, 1, None)
    _check(got, r)
    # both round the GeLU's result to bf16; the dispatched layer rounds the expert's output too
    tol = 2 * (6 * 2.0 ** -9 / math.sqrt(3.0) * r[4] + 2.0 ** -8 * r[3].abs()) + 2.0 ** -8 * r[3].abs() + 1e-6 * r[5]
    assert ((out.double() - got[0].double()).abs() <= tol).all()
