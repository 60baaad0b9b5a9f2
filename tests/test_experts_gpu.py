"""Tokens sorted by expert and back, the experts' products on the sorted rows, and their gradients, against plain 64-bit forms.

Tolerances.  A rounding to a type is off by at most half a step, relative to the value: bf16 2^-8, fp32 2^-24.  A sum of n terms
in fp32, in whatever order, is off by at most n 2^-24 times the sum of the terms' magnitudes (first order; products of bf16 are
exact in fp32, products of fp32 are rounded or fused, which the count n + 1 covers)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


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


def randn(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def plain_order(idx, E):
    """By Python lists, from the definition."""
    flat = idx.flatten().tolist()
    by = [[] for _ in range(E)]
    for v, e in enumerate(flat):
        if 0 <= e < E:
            by[e].append(v)
    offsets, rows = [0], []
    for b in by:
        rows += b
        offsets.append(len(rows))
    slot = [-1] * len(flat)
    for r, v in enumerate(rows):
        slot[v] = r
    t = lambda a: torch.tensor(a, dtype=I32, device="cuda")
    return t(offsets), t(slot).view_as(idx), t(rows + [-1] * (len(flat) - len(rows)))


def choices(g, T, K, E, kind):
    if kind == "none":
        return torch.full((K, T), -1, dtype=I32, device="cuda")
    if kind == "one":
        return torch.full((K, T), E - 1, dtype=I32, device="cuda")     # the same expert for every choice, too
    idx = torch.randint(0, E, (K, T), generator=g, device="cuda", dtype=I32)
    if kind == "bad":
        wild = torch.tensor([-1, -7, E, 2 ** 31 - 1, -2 ** 31], dtype=I32, device="cuda")
        at = torch.rand(K, T, generator=g, device="cuda") < 0.3
        idx = torch.where(at, wild[torch.randint(0, 5, (K, T), generator=g, device="cuda")], idx)
    return idx


def shifted(t, by=1):
    """The same values in memory that begins `by` elements behind an aligned address."""
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    flat[by:] = t.flatten()
    return flat[by:].view_as(t)


@pytest.mark.parametrize("T,K,E,kind", [(1, 1, 1, "any"), (1, 8, 3, "any"), (7, 2, 32, "bad"), (33, 3, 5, "one"), (64, 1, 1024, "any"), (100, 2, 8, "none"),
                                        (2731, 3, 64, "bad"), (8192, 1, 32, "any"), (8193, 1, 1024, "bad"), (30000, 2, 7, "any"), (70000, 4, 64, "bad"),
                                        (5000, 2, 1, "one")])
def test_order(X, B, T, K, E, kind):
    g = gen(T + K + E)
    idx = choices(g, T, K, E, kind)
    x = torch.zeros(T, 8, dtype=BF, device="cuda")
    xs, order = X.sort_rows(x, idx, E, want_load=True, want_rows=False)
    offsets, slot, inv = plain_order(idx, E)
    assert xs is None
    for got, want in zip(order, (offsets, slot, inv)):
        assert torch.equal(got, want)
    first = idx[0][(idx[0] >= 0) & (idx[0] < E)]
    assert torch.equal(order.load, torch.bincount(first.long(), minlength=E).to(I32))
    assert B.locmoe_device_flags() == 0


SHAPES = [(1, 1, 8, 1, "any"), (3, 8, 5, 4, "bad"), (5, 2, 2560, 4, "any"), (17, 3, 777, 7, "bad"), (300, 2, 96, 8, "any"), (64, 1, 64, 3, "none"),
          (1000, 4, 264, 16, "bad"), (4099, 2, 40, 8, "any"), (129, 1, 1234, 2, "one"), (2, 5, 9000, 3, "any"), (700, 3, 96, 8, "bad")]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,K,H,E,kind", SHAPES)
@pytest.mark.parametrize("shift", [0, 1])
def test_rows_there_and_back(X, B, T, K, H, E, kind, dt, shift):
    g = gen(T + H)
    move = lambda t: shifted(t, shift) if shift else t
    idx = choices(g, T, K, E, kind)
    x, res, dout = (move(randn(g, T, H, dtype=dt)) for _ in range(3))
    y, w = move(randn(g, K * T, H, dtype=dt)), torch.randn(K, T, generator=g, device="cuda")
    xs, order = X.sort_rows(x, idx, E)
    kept = int(order.offsets[-1])
    v = order.inv[:kept].long()
    assert torch.equal(xs[:kept], x[v % T]) and not xs[kept:].any()
    # what lies in rows without an assignment, or behind a weight without a row, is of no account
    y[kept:] = float("nan")
    w = torch.where(order.slot >= 0, w, float("inf"))
    terms = torch.zeros(K, T, H, dtype=torch.float64, device="cuda")
    terms.view(K * T, H)[v] = y[:kept].double() * w.flatten()[v].double()[:, None]
    for r, weights in ((None, w), (res, w), (res, None)):
        t = terms
        if weights is None:
            t = torch.zeros_like(terms)
            t.view(K * T, H)[v] = y[:kept].double()
        want = t.sum(0) + (0.0 if r is None else r.double())
        size = t.abs().sum(0) + (0.0 if r is None else r.double().abs())
        got = X.unsort_rows(y, order, weights, r)
        assert ((got.double() - want).abs() <= HALF[dt] * want.abs() + (K + 2) * 2.0 ** -24 * size).all()
    # gradients
    dy, dw = X.unsort_rows_grad(dout, order, w, y)
    want = dout[v % T].double() * w.flatten()[v].double()[:, None]
    assert ((dy[:kept].double() - want).abs() <= (HALF[dt] + 2.0 ** -24) * want.abs()).all() and not dy[kept:].any()
    want = torch.zeros(K * T, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    prod = dout[v % T].double() * y[:kept].double()
    want[v], size[v] = prod.sum(1), prod.abs().sum(1)
    assert ((dw.flatten().double() - want).abs() <= (H + 2) * 2.0 ** -24 * size).all()
    only, none = X.unsort_rows_grad(dout, order)
    assert none is None and torch.equal(only[:kept], dout[v % T]) and not only[kept:].any()
    none, dw2 = X.unsort_rows_grad(dout, order, w, y, want_dy=False)
    assert none is None and torch.equal(dw2, dw)
    dx, none = X.sort_rows_grad(y, order)
    t = torch.zeros(K, T, H, dtype=torch.float64, device="cuda")
    t.view(K * T, H)[v] = y[:kept].double()
    assert none is None
    assert ((dx.double() - t.sum(0)).abs() <= HALF[dt] * t.sum(0).abs() + (K + 1) * 2.0 ** -24 * t.abs().sum(0)).all()
    assert B.locmoe_device_flags() == 0


def router64(x, idx, dw, eps, dp):
    """dG, G, p and the terms' size of the router's gradient."""
    T, E = x.shape[0], dp.numel()
    G = x.double().view(T, E, -1).mean(2) + eps.double()
    p = torch.softmax(G.clamp_min(0.0), 1)
    q = dp.double()[None].repeat(T, 1)
    size = dp.double().abs()[None].repeat(T, 1)
    for k in range(idx.shape[0]):
        t = torch.nonzero((idx[k] >= 0) & (idx[k] < E)).squeeze(1)
        q[t, idx[k, t].long()] += dw[k, t].double()
        size[t, idx[k, t].long()] += dw[k, t].double().abs()
    m = (p * q).sum(1, keepdim=True)
    return torch.where(G > 0, p * (q - m), 0.0), G, p, size + (p * size).sum(1, keepdim=True)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,K,H,E,kind", [(1, 1, 8, 1, "any"), (9, 2, 2560, 32, "any"), (33, 3, 777, 21, "bad"), (65, 1, 5120, 64, "any"), (50, 8, 1024, 1024, "any"),
                                          (700, 2, 1000, 4, "bad"), (2500, 4, 128, 32, "none"), (40, 1, 12288, 3, "any"), (31, 3, 1236, 6, "bad"),
                                          (6000, 2, 96, 24, "any"), (7001, 1, 72, 8, "any"), (6500, 2, 256, 64, "bad"), (9000, 3, 189, 21, "any"),
                                          (6400, 4, 256, 32, "none"), (6350, 8, 100, 10, "bad"), (6321, 1, 768, 3, "any")])
def test_router_gradient(X, B, T, K, H, E, kind, dt):
    g = gen(T * 3 + H)
    idx = choices(g, T, K, E, kind)
    x, dxs = randn(g, T, H, dtype=dt), randn(g, K * T, H, dtype=dt)
    dw, dp, eps = torch.randn(K, T, generator=g, device="cuda"), torch.randn(E, generator=g, device="cuda"), randn(g, E, std=0.3)
    _, order = X.sort_rows(x, idx, E, want_rows=False)
    kept = int(order.offsets[-1])
    dxs[kept:] = float("nan")
    dG, G, p, size = router64(x, idx, dw, eps, dp)
    n = H // E
    # G is off by `off`: a sum of n terms in fp32, scaled and shifted.  p follows with 2 off (its own exponent and the sum's), the
    # exponential (2 steps), the sum over E and the division; q - m has K + E + 2 roundings of its terms
    off = (n + 3) * 2.0 ** -24 * (x.double().abs().view(T, E, -1).mean(2) + eps.double().abs())
    rel = 2 * off.amax(1, keepdim=True) + (E + 8) * 2.0 ** -24
    tol = p * size * (2 * rel + (K + E + 4) * 2.0 ** -24)
    clear = G.abs() > off                       # where the sign of G is beyond doubt
    assert clear.double().mean() > 0.99
    deps_tol = (tol + torch.where(clear, 0.0, p * size)).sum(0) + (T + 2) * 2.0 ** -24 * dG.abs().sum(0)
    t = torch.zeros(K, T, H, dtype=torch.float64, device="cuda")
    v = order.inv[:kept].long()
    t.view(K * T, H)[v] = dxs[:kept].double()
    spread = lambda a: (a / n)[:, :, None].expand(T, E, n).reshape(T, H)
    for d in (dxs, None):
        rows, mags = (t.sum(0), t.abs().sum(0)) if d is not None else (0.0, 0.0)
        dx, deps = X.sort_rows_grad(d, order, x, idx, dw, eps, dp)
        want = rows + spread(dG)
        bound = HALF[dt] * want.abs() + (1 + HALF[dt]) * (spread(tol) + (K + 2) * 2.0 ** -24 * (mags + spread(dG.abs())))
        bad = (dx.double() - want).abs() > bound
        assert not (bad & spread(clear.double() * n).bool()).any()
        assert ((deps.double() - dG.sum(0)).abs() <= deps_tol).all()
    # without scores, bias or loss
    zero = torch.zeros(E, device="cuda")
    for kw in (dict(dp=dp), dict(idx_k=idx, dw=dw)):
        dG, G, p, size = router64(x, idx, kw.get("dw", torch.zeros_like(dw)), zero, kw.get("dp", zero))
        dx, none = X.sort_rows_grad(None, order, x, want_deps=False, **kw)
        tol = p * size * (2 * rel + (K + E + 4) * 2.0 ** -24)
        bad = (dx.double() - spread(dG)).abs() > HALF[dt] * spread(dG).abs() + 2 * spread(tol)
        assert none is None and not (bad & (spread(G.abs()) * n > spread(off) * n)).any()
    assert B.locmoe_device_flags() == 0


def test_router_gradient_against_differences(X, B):
    """The loss sum(c * w_k) + sum_t,e dp_e p_e of the forward pass in 64 bits, moved along random directions."""
    g = gen(5)
    T, H, E, K, h = 40, 96, 8, 2, 1e-5
    x, c, dp = randn(g, T, H), torch.randn(K, T, generator=g, device="cuda"), torch.randn(E, generator=g, device="cuda")
    eps = randn(g, E, std=0.1)
    p0 = torch.softmax((x.double().view(T, E, -1).mean(2) + eps.double()).clamp_min(0), 1)
    idx = p0.topk(K, 1).indices.t().contiguous().to(I32)

    def loss(x64, eps64):
        p = torch.softmax((x64.view(T, E, -1).mean(2) + eps64).clamp_min(0), 1)
        return (c.double() * p.gather(1, idx.t().long()).t()).sum() + (p * dp.double()).sum()
    _, order = X.sort_rows(x, idx, E, want_rows=False)
    dx, deps = X.sort_rows_grad(None, order, x, idx, c, eps, dp)
    for seed in range(4):
        d, de = randn(gen(seed), T, H).double(), randn(gen(seed + 9), E).double()
        diff = (loss(x.double() + h * d, eps.double() + h * de) - loss(x.double() - h * d, eps.double() - h * de)) / (2 * h)
        want = (dx.double() * d).sum() + (deps.double() * de).sum()
        size = (dx.double() * d).abs().sum() + (deps.double() * de).abs().sum()
        # differences of a smooth function are off by h^2 of its third derivative (of order 1); a G within h |d| of zero
        # changes sides, which costs at most its own term: T E groups, a chance of 1e-5 each
        assert abs(float(diff - want)) <= 1e-5 * float(size)


ACT64 = dict(none=lambda v: v, relu=lambda v: v.clamp_min(0), gelu=lambda v: v * torch.special.ndtr(v), silu=lambda v: v * torch.sigmoid(v))


def slope64(v, act):
    if act == "relu":
        return (v > 0).double()
    if act == "gelu":
        return torch.special.ndtr(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        q = torch.sigmoid(v)
        return q * (1 + v * (1 - q))
    return torch.ones_like(v)


def ragged(counts, lost=0):
    o = torch.tensor([0] + counts, device="cuda").cumsum(0).to(I32)
    return o, int(o[-1]) + lost


# rows per expert: one row, groups that end in every part of a tile, experts without rows (first, last, between), one that has all
GROUPS = [([1], 0), ([0, 2, 0, 0, 1], 0), ([3, 0, 64, 65, 127, 128, 129, 16, 17, 0], 5), ([0, 0, 700, 0], 0), ([0, 0, 0], 9), ([5] * 40, 1), ([300, 1, 257], 0)]
SIZES = [(8, 8), (64, 256), (72, 264), (200, 40), (1560, 520), (520, 2056)]


@pytest.mark.parametrize("counts,lost", GROUPS)
@pytest.mark.parametrize("IN,OUT", SIZES)
def test_products(X, B, counts, lost, IN, OUT):
    offsets, R = ragged(counts, lost)
    E, g, o = len(counts), gen(R + IN), offsets.tolist()
    x, w = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF, std=IN ** -0.5)
    x[o[-1]:] = float("nan")                              # rows behind the last group are of no account
    bias, res = randn(g, E, OUT), randn(g, R, OUT, dtype=BF)
    z64, size = torch.zeros(R, OUT, dtype=torch.float64, device="cuda"), torch.zeros(R, OUT, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = o[e], o[e + 1]
        z64[a:b], size[a:b] = x[a:b].double() @ w[e].double().t(), x[a:b].double().abs() @ w[e].double().abs().t()
    by_row = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.tensor(counts, device="cuda"))
    kept = o[-1]
    for act, bi, r, want_z in (("none", None, None, False), ("gelu", bias, None, True), ("silu", bias, res, False), ("relu", None, res, True)):
        v, off = z64.clone(), (IN + 2) * 2.0 ** -24 * size
        if bi is not None:
            v[:kept] += bi[by_row].double()
            off[:kept] += 2.0 ** -24 * bi[by_row].double().abs()
        y, z = X.expert_linear(x, w, offsets, bi, act, r, want_z)
        # the slopes are below 1.13 (GeLU) and 1.1 (SiLU); the approximations' error: 1.5e-7 |v| for erf, a few 2^-22 |v| for the
        # exponential and the reciprocal
        want, tol = ACT64[act](v), 1.13 * off + 2e-6 * v.abs()
        if r is not None:
            want = want + r.double()
            tol = tol + 2.0 ** -24 * want.abs()
        want[kept:] = 0.0
        assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * tol)[:kept].all() and not y[kept:].any()
        assert (z is not None) == want_z
        if want_z:
            assert ((z.double() - v).abs() <= 2.0 ** -8 * v.abs() + (1 + 2.0 ** -8) * off)[:kept].all() and not z[kept:].any()
    # gradients
    dy, zin = randn(g, R, OUT, dtype=BF), randn(g, R, IN, dtype=BF)
    dy[kept:], zin[kept:] = float("inf"), float("nan")
    dx64, size = torch.zeros(R, IN, dtype=torch.float64, device="cuda"), torch.zeros(R, IN, dtype=torch.float64, device="cuda")
    dw64, wsize = torch.zeros(E, OUT, IN, dtype=torch.float64, device="cuda"), torch.zeros(E, OUT, IN, dtype=torch.float64, device="cuda")
    db64, bsize = torch.zeros(E, OUT, dtype=torch.float64, device="cuda"), torch.zeros(E, OUT, dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = o[e], o[e + 1]
        d, xe = dy[a:b].double(), x[a:b].double()
        dx64[a:b], size[a:b] = d @ w[e].double(), d.abs() @ w[e].double().abs()
        dw64[e], wsize[e] = d.t() @ xe, d.abs().t() @ xe.abs()
        db64[e], bsize[e] = d.sum(0), d.abs().sum(0)
    rows = max(counts) + 2
    for act, dwt in (("none", F32), ("gelu", BF), ("silu", F32), ("relu", BF)):
        zi = None if act == "none" else zin
        dx, dw, db = X.expert_linear_grad(dy, x, w, offsets, zi, act, want_db=True, dw_dtype=dwt)
        f = slope64(zin.double(), act)
        want, tol = dx64 * f, (OUT + 2) * 2.0 ** -24 * size * f.abs() + 4e-6 * dx64.abs() * (1 + zin.double().abs())
        assert ((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * tol)[:kept].all() and not dx[kept:].any()
        assert dw.dtype == dwt and ((dw.double() - dw64).abs() <= HALF[dwt] * dw64.abs() + (1 + 2.0 ** -8) * rows * 2.0 ** -24 * wsize).all()
        assert ((db.double() - db64).abs() <= rows * 2.0 ** -24 * bsize).all()
    assert B.locmoe_device_flags() == 0


@pytest.mark.parametrize("counts,lost", [([3, 5, 2], 1), ([200, 100, 130, 0, 7], 0), ([130] * 64, 3)])
def test_an_expert_with_infinities_disturbs_no_other(X, counts, lost):
    offsets, R = ragged(counts, lost)
    E, IN, OUT, g, o = len(counts), 136, 264, gen(R), offsets.tolist()
    x, w, dy, z = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF), randn(g, R, OUT, dtype=BF), randn(g, R, IN, dtype=BF)
    clean = (X.expert_linear(x, w, offsets, act="gelu")[0], *X.expert_linear_grad(dy, x, w, offsets, z, "gelu", want_db=True))
    a, b = o[1], o[2]
    x[a:b], dy[a:b], z[a:b], w[1] = float("nan"), float("inf"), float("-inf"), float("nan")
    dirty = (X.expert_linear(x, w, offsets, act="gelu")[0], *X.expert_linear_grad(dy, x, w, offsets, z, "gelu", want_db=True))
    for i, (c, d) in enumerate(zip(clean, dirty)):
        rows = (slice(0, a), slice(b, R)) if i < 2 else (slice(0, 1), slice(2, E))
        for r in rows:
            assert torch.equal(c[r], d[r])
        assert not d[slice(a, b) if i < 2 else 1].isfinite().any()


def test_long_groups_and_every_way_of_dealing_the_work(X, B):
    """Few tiles with a long reduction (runs within a tile), many tiles (dealt one by one), in all three products."""
    for seed, (counts, IN, OUT) in enumerate([([20000, 0, 3], 16, 24), ([2], 8192, 520), ([40, 9], 6000, 2048), ([2100, 900, 4000, 77], 512, 10240)]):
        offsets, R = ragged(counts)
        E, g, o = len(counts), gen(seed), offsets.tolist()
        x, w, dy = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF, std=IN ** -0.5), randn(g, R, OUT, dtype=BF)
        y, _ = X.expert_linear(x, w, offsets)
        dx, dw, db = X.expert_linear_grad(dy, x, w, offsets, want_db=True, dw_dtype=F32)
        again = X.expert_linear_grad(dy, x, w, offsets, want_db=True, dw_dtype=F32)
        for a, b in zip((y, dx, dw, db), (X.expert_linear(x, w, offsets)[0], *again)):
            assert torch.equal(a, b)                                # sums have a fixed order
        for e in range(E):
            s = slice(o[e], o[e + 1])
            xe, we, de = x[s].double(), w[e].double(), dy[s].double()
            for got, want, size, n, half in ((y[s], xe @ we.t(), xe.abs() @ we.abs().t(), IN, 2.0 ** -8), (dx[s], de @ we, de.abs() @ we.abs(), OUT, 2.0 ** -8),
                                             (dw[e], de.t() @ xe, de.abs().t() @ xe.abs(), counts[e], 2.0 ** -24)):
                assert ((got.double() - want).abs() <= half * want.abs() + (n + 3) * 2.0 ** -24 * (1 + half) * size).all()
    assert B.locmoe_device_flags() == 0


@pytest.mark.parametrize("counts,lost,IN,OUT", [([2300], 0, 9208, 8200), ([4000, 129, 0, 1, 9000, 257, 5300], 11, 1544, 6600), ([9000, 0, 11001], 300, 1544, 2856)])
def test_many_tiles_of_long_groups(X, B, counts, lost, IN, OUT):
    """Sizes at which a tile has two accumulators: groups that end in either half, the same sums again, a bias's gradient of both."""
    offsets, R = ragged(counts, lost)
    E, g, o = len(counts), gen(R), offsets.tolist()
    x, w, dy = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF, std=IN ** -0.5), randn(g, R, OUT, dtype=BF)
    bias, zin = randn(g, E, OUT), randn(g, R, IN, dtype=BF)
    for t in (x, dy, zin):
        t[o[-1]:] = float("nan")
    y, z = X.expert_linear(x, w, offsets, bias, "relu", want_z=True)
    dx, dw, db = X.expert_linear_grad(dy, x, w, offsets, zin, "relu", want_db=True)
    again = X.expert_linear_grad(dy, x, w, offsets, zin, "relu", want_db=True)
    assert all(torch.equal(a, b) for a, b in zip((y, z, dx, dw, db), (*X.expert_linear(x, w, offsets, bias, "relu", want_z=True), *again)))
    for t in (y, z, dx):
        assert not t[o[-1]:].any()
    for e in range(E):
        s = slice(o[e], o[e + 1])
        xe, we, de = x[s].double(), w[e].double(), dy[s].double()
        v = xe @ we.t() + bias[e].double()
        f = (zin[s] > 0).double()
        vsize = xe.abs() @ we.abs().t() + bias[e].double().abs()
        for got, want, size, n, half in ((z[s], v, vsize, IN, 2.0 ** -8), (y[s], v.clamp_min(0), vsize, IN, 2.0 ** -8),
                                         (dx[s], de @ we * f, de.abs() @ we.abs(), OUT, 2.0 ** -8),
                                         (dw[e], de.t() @ xe, de.abs().t() @ xe.abs(), counts[e], 2.0 ** -8),
                                         (db[e], de.sum(0), de.abs().sum(0), counts[e], 2.0 ** -24)):
            assert ((got.double() - want).abs() <= half * want.abs() + (n + 3) * 2.0 ** -24 * (1 + half) * size).all()
        del xe, we, de, v, f, vsize, got, want, size
    assert B.locmoe_device_flags() == 0


def test_offsets_that_make_no_sense_touch_nothing_else(X, B):
    """Offsets that descend or leave the rows: unspecified rows, and no access beyond the arrays."""
    g = gen(1)
    R, IN, OUT, E = 70, 72, 136, 4
    x, w, dy = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF), randn(g, R, OUT, dtype=BF)
    for o in ([0, 90, 20, 2 ** 31 - 1, 70], [-5, -2 ** 31, 30, 10, 500], [70, 70, 0, 0, -1], [2 ** 31 - 1] * 5):
        offsets = torch.tensor(o, dtype=I32, device="cuda")
        X.expert_linear(x, w, offsets, act="gelu", want_z=True)
        X.expert_linear_grad(dy, x, w, offsets, want_db=True)
    torch.cuda.synchronize()
    assert B.locmoe_device_flags() == 0


FEW = [([1], 0), ([0, 1, 0, 0, 1], 0), ([2, 1], 1), ([4], 0), ([0, 3, 0, 1], 0), ([1] * 8, 0), ([8], 0), ([5, 0, 2], 1), ([0] * 40 + [1, 1] + [0] * 40, 0), ([0, 0], 3)]


@pytest.mark.parametrize("counts,lost", FEW)
@pytest.mark.parametrize("IN,OUT", [(8, 8), (264, 72), (1000, 1544), (10240, 24), (2056, 4104)])
def test_a_few_rows(X, B, counts, lost, IN, OUT):
    """Single tokens and a few more, with all that may come with the product."""
    offsets, R = ragged(counts, lost)
    E, g, kept = len(counts), gen(R + IN), sum(counts)
    x, w = randn(g, R, IN, dtype=BF), randn(g, E, OUT, IN, dtype=BF, std=IN ** -0.5)
    bias, res = randn(g, E, OUT), randn(g, R, OUT, dtype=BF)
    x[kept:] = float("nan")
    e_of = torch.repeat_interleave(torch.arange(E), torch.tensor(counts)).cuda()
    v = torch.bmm(w[e_of].double(), x[:kept].double()[:, :, None])[:, :, 0]
    size = torch.bmm(w[e_of].double().abs(), x[:kept].double().abs()[:, :, None])[:, :, 0]
    for act, bi, r, want_z in (("none", None, None, False), ("gelu", bias, None, True), ("silu", bias, res, True), ("relu", None, res, False)):
        u = v if bi is None else v + bi[e_of].double()
        off = (IN + 3) * 2.0 ** -24 * (size if bi is None else size + bi[e_of].double().abs())
        y, z = X.expert_linear(x, w, offsets, bi, act, r, want_z)
        want, tol = ACT64[act](u), 1.13 * off + 2e-6 * u.abs()              # slopes and approximations as above
        if r is not None:
            want = want + r[:kept].double()
            tol = tol + 2.0 ** -24 * want.abs()
        assert ((y[:kept].double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * tol).all() and not y[kept:].any()
        assert (z is not None) == want_z
        if want_z:
            assert ((z[:kept].double() - u).abs() <= 2.0 ** -8 * u.abs() + (1 + 2.0 ** -8) * off).all() and not z[kept:].any()
    assert B.locmoe_device_flags() == 0


def test_a_few_rows_and_offsets_of_all_kinds(X):
    """A slice of the offsets: zeros before and behind.  Offsets that make no sense: no access beyond the arrays."""
    g = gen(5)
    x, w = randn(g, 7, 136, dtype=BF), randn(g, 3, 40, 136, dtype=BF)
    y, z = X.expert_linear(x, w, torch.tensor([0, 2, 3, 3, 5, 7], dtype=I32, device="cuda")[1:5], act="gelu", want_z=True)
    for t in (y, z):
        assert not t[:2].any() and not t[5:].any() and t[2:5].any(1).all()
    for o in ([0, 90, -20, 2 ** 31 - 1], [7, 0, 7, 0], [-5, -2 ** 31, 3, 1], [2 ** 31 - 1] * 4):
        X.expert_linear(x, w, torch.tensor(o, dtype=I32, device="cuda"), act="gelu", want_z=True)
    torch.cuda.synchronize()


@pytest.mark.parametrize("counts,lost", GROUPS + [([3000, 0, 1, 700], 9)])
@pytest.mark.parametrize("OUT", [8, 72, 520])
def test_the_gradient_of_the_bias_alone(X, counts, lost, OUT):
    offsets, R = ragged(counts, lost)
    dy, w = randn(gen(OUT), R, OUT, dtype=BF), torch.zeros(len(counts), OUT, 8, dtype=BF, device="cuda")
    dy[int(offsets[-1]):] = float("nan")
    dx, dw, db = X.expert_linear_grad(dy, None, w, offsets, want_dx=False, want_dw=False, want_db=True)
    assert dx is None and dw is None
    for e, d in enumerate(dy[:int(offsets[-1])].double().split(counts)):
        assert ((db[e].double() - d.sum(0)).abs() <= counts[e] * 2.0 ** -24 * d.abs().sum(0)).all()


@pytest.mark.parametrize("counts,lo,hi", [([70, 3, 130, 0, 9], 1, 3), ([5, 0, 300, 20], 2, 3), ([40, 50, 60], 1, 1)])
def test_a_part_of_the_experts(X, B, counts, lo, hi):
    """A slice of the offsets with its experts' weights: their rows as in the whole, zeros in all others."""
    g = gen(7)
    offsets, R = ragged(counts, 2)
    E, a, b = hi - lo + 1, int(offsets[lo]), int(offsets[hi + 1])
    part = offsets[lo:hi + 2]
    x, w, dy, bias = randn(g, R, 200, dtype=BF), randn(g, E, 264, 200, dtype=BF), randn(g, R, 264, dtype=BF), randn(g, E, 264)
    for t in (x, dy):
        t[:a], t[b:] = float("nan"), float("inf")
    y, z = X.expert_linear(x, w, part, bias, "silu", want_z=True)
    dx, dw, db = X.expert_linear_grad(dy, x, w, part, want_db=True, dw_dtype=F32)
    own = part - a
    y1, z1 = X.expert_linear(x[a:b].clone(), w, own, bias, "silu", want_z=True)
    dx1, dw1, db1 = X.expert_linear_grad(dy[a:b].clone(), x[a:b].clone(), w, own, want_db=True, dw_dtype=F32)
    # the same sums, in another order at most: (terms + 3) 2^-24 of the sum of the magnitudes for each, the slope of SiLU 1.1; and
    # bf16's rounding of each.  A row's sum of magnitudes is below its norms' product.
    for got, want, left, terms in ((y, y1, x, 200), (z, z1, x, 200), (dx, dx1, dy, 264)):
        norm = left[a:b].float().norm(dim=1, keepdim=True) * w.float().norm(dim=2 if left is x else 1).max() + bias.abs().max()
        assert ((got[a:b].float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2 * 1.13 * (terms + 3) * 2.0 ** -24 * norm).all()
        assert not got[:a].any() and not got[b:].any()
    magnitudes = [(dy[s:t].float().abs(), x[s:t].float().abs()) for s, t in zip(part[:-1].tolist(), part[1:].tolist())]
    tol = 2 * (max(counts) + 3) * 2.0 ** -24
    assert ((dw - dw1).abs() <= tol * torch.stack([d.t() @ v for d, v in magnitudes])).all()
    assert ((db - db1).abs() <= tol * torch.stack([d.sum(0) for d, _ in magnitudes])).all()
    assert B.locmoe_device_flags() == 0


def test_residual_may_be_the_output(X, B):
    g = gen(2)
    offsets, R = ragged([4, 0, 200, 3])
    x, w, y = randn(g, R, 64, dtype=BF), randn(g, 4, 264, 64, dtype=BF), randn(g, R, 264, dtype=BF)
    want, _ = X.expert_linear(x, w, offsets, residual=y)
    shape = B.Shape(R, 64, 4, 1, 1, B.BF16, 0)
    ws = torch.empty(B.locmoe_expert_linear_bytes(shape, 264), dtype=torch.uint8, device="cuda")
    B.locmoe_expert_linear(shape, 264, x, w, offsets, y, ws, residual=y)
    assert torch.equal(y, want)
    out = randn(g, 5, 40)
    _, order = X.sort_rows(out, choices(g, 5, 2, 3, "any"), 3, want_rows=False)
    rows, wk = randn(g, 10, 40), randn(g, 2, 5)
    want = X.unsort_rows(rows, order, wk, out)
    B.locmoe_unsort(B.Shape(5, 40, 3, 1, 1, B.F32, 0), 2, rows, order.slot, out, wk, out)
    assert torch.equal(out, want)


def layer_inputs(g, T, H, F, E, K, dt=BF):
    return dict(x=randn(g, T, H, dtype=dt), w_in=randn(g, E, F, H, dtype=dt, std=0.1), w_out=randn(g, E, H, F, dtype=dt, std=0.1), b_in=randn(g, E, F, std=0.1),
                b_out=randn(g, E, H, std=0.1), eps=randn(g, E, std=0.1), residual=randn(g, T, H, dtype=dt))


def layer64(p, idx, act, alpha, K):
    """The layer in 64 bits for given choices, by autograd on dense products."""
    x, E = p["x"], p["w_in"].shape[0]
    T = x.shape[0]
    prob = torch.softmax((x.view(T, E, -1).mean(2) + p["eps"]).clamp_min(0), 1)
    out = p["residual"]
    for k in range(K):
        e = idx[k].long()
        a = ACT64[act](torch.einsum("th,tfh->tf", x, p["w_in"][e]) + p["b_in"][e])
        y = torch.einsum("tf,thf->th", a, p["w_out"][e]) + p["b_out"][e]
        out = out + prob.gather(1, e[:, None]) * y
    f = torch.bincount(idx[0].long(), minlength=E).double() / T
    return out, alpha * E * (f * prob.mean(0)).sum()


@pytest.mark.parametrize("T,H,F,E,K,act", [(1, 64, 128, 4, 1, "gelu"), (50, 64, 72, 8, 2, "silu"), (300, 128, 264, 4, 3, "relu"), (130, 96, 64, 3, 1, "none")])
def test_the_layer_and_its_gradient(X, T, H, F, E, K, act):
    g = gen(T)
    p = layer_inputs(g, T, H, F, E, K)
    leaves = {k: v.clone().requires_grad_() for k, v in p.items()}
    c, alpha = randn(g, T, H, dtype=BF), 0.01
    out, aux = X.moe_layer(leaves["x"], leaves["w_in"], leaves["w_out"], K, leaves["b_in"], leaves["b_out"], leaves["eps"], act, leaves["residual"], alpha)
    idx = X.RouteSort.apply(p["x"], p["eps"], E, K, 0.0)[3]
    ref = {k: v.double().requires_grad_() for k, v in p.items()}
    out64, aux64 = layer64(ref, idx, act, alpha, K)
    ((out.float() * c.float()).sum() + 3.0 * aux).backward()
    ((out64 * c.double()).sum() + 3.0 * aux64).backward()
    assert abs(float(aux) - float(aux64)) <= 1e-5 * float(aux64)
    # bf16 roundings on the way (rows, the activation, its gradient, the outputs): each 2^-8 at most of an element, independent, so
    # that norms differ by a few times 2^-8 / sqrt(3); where an activation is near its kink nothing jumps by more than that
    for name, got, want in [("out", out, out64)] + [(k, leaves[k].grad, ref[k].grad) for k in p]:
        assert got.dtype == (out if name == "out" else leaves[name]).dtype
        assert float((got.double() - want).norm()) <= 4 * 2.0 ** -8 * float(want.norm()) + 1e-6, name


def test_parts_that_need_no_gradient_get_none(X):
    g = gen(3)
    p = layer_inputs(g, 20, 64, 72, 4, 1)
    for need in ("x", "w_in", "w_out", "b_in", "b_out", "eps", "residual"):
        leaves = {k: v.clone().requires_grad_(k == need) for k, v in p.items()}
        out, aux = X.moe_layer(leaves["x"], leaves["w_in"], leaves["w_out"], 2, leaves["b_in"], leaves["b_out"], leaves["eps"], "gelu", leaves["residual"], 0.0)
        assert aux is None
        out.float().sum().backward()
        for k, v in leaves.items():
            assert (v.grad is not None) == (k == need)
            assert k != need or bool(v.grad.isfinite().all())
    x = p["x"].clone().requires_grad_()
    loss = X.moe_layer(x, p["w_in"], p["w_out"], eps=p["eps"], alpha=0.1)[1]     # the balance loss alone
    loss.backward()
    assert bool(x.grad.isfinite().all()) and bool(x.grad.any())
    with pytest.raises(RuntimeError):
        y = X.Unsort.apply(x, None, None, *X.RouteSort.apply(x.detach(), None, 4, 1, 0.0)[4:])
        d = torch.autograd.grad(y.float().sum(), x, create_graph=True)[0]
        torch.autograd.grad(d.float().sum(), x)


def test_tensors_of_another_device_are_refused(X, monkeypatch):
    g = gen(4)
    p = layer_inputs(g, 20, 64, 72, 4, 1)
    args = (p["x"], p["w_in"], p["w_out"], 2)
    for bad in (dict(eps=p["eps"].cpu()), dict(eps=torch.zeros(5, device="cuda"))):
        with pytest.raises(ValueError):
            X.moe_layer(*args, **bad)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)            # as if the tensors were on a device that is not current
    with pytest.raises(ValueError, match="not the current"):
        X.moe_layer(*args)
    with pytest.raises(ValueError, match="not the current"):
        X.RouteSort.apply(p["x"], None, 4, 1, 0.0)


def test_nothing_to_do(X):
    x, w = torch.zeros(0, 64, dtype=BF, device="cuda"), torch.ones(3, 8, 64, dtype=BF, device="cuda")
    xs, order = X.sort_rows(x, torch.zeros(2, 0, dtype=I32, device="cuda"), 3, want_load=True)
    assert xs.shape == (0, 64) and order.offsets.tolist() == [0] * 4 and order.load.tolist() == [0] * 3
    assert X.sort_rows_grad(xs, order, x, dp=torch.ones(3, device="cuda"))[1].tolist() == [0.0] * 3
    assert X.unsort_rows(xs, order).shape == (0, 64)
    y, z = X.expert_linear(xs, w, order.offsets, want_z=True)
    assert y.shape == z.shape == (0, 8)
    dx, dw, db = X.expert_linear_grad(y, xs, w, order.offsets, want_db=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    leaf = torch.zeros(0, 64, dtype=BF, device="cuda", requires_grad=True)
    w2 = torch.ones(4, 8, 64, dtype=BF, device="cuda", requires_grad=True)
    out, aux = X.moe_layer(leaf, w2, w2.detach().transpose(1, 2).contiguous(), 2, alpha=0.1)
    (out.float().sum() + aux).backward()
    assert leaf.grad.shape == (0, 64) and not w2.grad.any()


def step(X, p, K=2):
    """Order, rows, both products, the way back and all gradients: a list of tensors."""
    E = p["w_in"].shape[0]
    xs, order = X.sort_rows(p["x"], p["idx"], E)
    a, z = X.expert_linear(xs, p["w_in"], order.offsets, p["b_in"], "gelu", want_z=True)
    y, _ = X.expert_linear(a, p["w_out"], order.offsets, p["b_out"])
    out = X.unsort_rows(y, order, p["w_k"], p["residual"])
    dy, dwk = X.unsort_rows_grad(out, order, p["w_k"], y)
    dz, dwo, dbo = X.expert_linear_grad(dy, a, p["w_out"], order.offsets, z, "gelu", want_db=True)
    dxs, dwi, dbi = X.expert_linear_grad(dz, xs, p["w_in"], order.offsets, want_db=True)
    dx, deps = X.sort_rows_grad(dxs, order, p["x"], p["idx"], dwk, p["eps"])
    return [xs, *order[:3], a, z, y, out, dy, dwk, dz, dwo, dbo, dxs, dwi, dbi, dx, deps]


def step_inputs(seed, T=37, H=64, F=136, E=8, K=2):
    g = gen(seed)
    return dict(layer_inputs(g, T, H, F, E, K), idx=choices(g, T, K, E, "bad"), w_k=torch.rand(K, T, generator=g, device="cuda"))


def test_captured_and_replayed(X):
    """Two graphs of whole steps, replayed in turn with inputs that change, an eager step between."""
    ps = [step_inputs(1), step_inputs(2, T=300, F=264)]
    graphs = []
    for p in ps:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            step(X, p)
        torch.cuda.current_stream().wait_stream(s)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = step(X, p)
        graphs.append((gr, out))
    for seed in (5, 6):
        for i, p in enumerate(ps):
            new = step_inputs(seed) if i == 0 else step_inputs(seed, T=300, F=264)
            for k in p:
                p[k].copy_(new[k])
        for gr, _ in graphs:
            gr.replay()
        want = [step(X, p) for p in ps]
        torch.cuda.synchronize()
        for (_, got), w in zip(graphs, want):
            assert all(torch.equal(a, b) for a, b in zip(got, w))


def test_two_streams_at_once(X):
    ps = [step_inputs(7, T=500, F=264), step_inputs(8, T=900, H=128, F=512)]
    want = [step(X, p) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(step(X, ps[i]))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for r in g:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


def test_stream_argument(X):
    p = step_inputs(9, T=200)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    E = 8
    xs, order = X.sort_rows(p["x"], p["idx"], E, stream=s)
    a, z = X.expert_linear(xs, p["w_in"], order.offsets, p["b_in"], "gelu", want_z=True, stream=s)
    y, _ = X.expert_linear(a, p["w_out"], order.offsets, p["b_out"], stream=s.cuda_stream)
    out = X.unsort_rows(y, order, p["w_k"], p["residual"], stream=s)
    dy, dwk = X.unsort_rows_grad(out, order, p["w_k"], y, stream=s)
    dz, dwo, dbo = X.expert_linear_grad(dy, a, p["w_out"], order.offsets, z, "gelu", want_db=True, stream=s)
    dx, deps = X.sort_rows_grad(X.expert_linear_grad(dz, xs, p["w_in"], order.offsets, want_dw=False, stream=s)[0], order, p["x"], p["idx"], dwk, p["eps"], stream=s)
    torch.cuda.synchronize()
    want = step(X, p)
    for got, i in ((xs, 0), (a, 4), (out, 7), (dwk, 9), (dz, 10), (dwo, 11), (dx, 16), (deps, 17)):
        assert torch.equal(got, want[i])


def test_rows_beyond_32_bit_offsets(X):
    """More than 2^31 elements in the sorted rows: the last rows are where they belong."""
    T, H, K, E = 270000, 8192, 1, 2
    x = torch.zeros(T, H, dtype=BF, device="cuda")
    x[-1], x[0] = 3.0, 1.0
    idx = torch.zeros(K, T, dtype=I32, device="cuda")
    idx[0, 0] = 1                                              # token 0 goes last
    xs, order = X.sort_rows(x, idx, E)
    assert bool((xs[T - 1] == 1.0).all()) and bool((xs[T - 2] == 3.0).all()) and not xs[:T - 2].any()
    out = X.unsort_rows(xs, order)
    assert torch.equal(out, x)
    del out
    dy, dw = X.unsort_rows_grad(x, order, y=xs)
    assert torch.equal(dy, xs) and dw[0, 0] == H and dw[0, -1] == 9.0 * H and not dw[0, 1:-1].any()
    del dy
    w = torch.zeros(E, 8, H, dtype=BF, device="cuda")
    w[1, 3], w[0, 5] = 1.0, 2.0 ** -4
    y, _ = X.expert_linear(xs, w, order.offsets)
    assert y[T - 1].tolist() == [0, 0, 0, H, 0, 0, 0, 0] and y[T - 2].tolist() == [0, 0, 0, 0, 0, 3 * H / 16, 0, 0]
    dx, dwt, _ = X.expert_linear_grad(y, xs, w, order.offsets, dw_dtype=F32)
    assert bool((dx[T - 1] == H).all()) and bool((dx[T - 2] == 3 * H / 256).all()) and not dx[:T - 2].any()
    assert bool((dwt[1, 3] == H).all()) and bool((dwt[0, 5] == 9 * H / 16).all())
