"""The fused block norms and their gradient on the GPU against a plain implementation in 64 bits.

Tolerances: fp32 sums of up to H terms in trees of at most ~H/32 sequential adds and two products after them, so a
relative error of 2e-6 of a value's own scale covers fp32 outputs (column sums: their root-sum-square scale); bf16
outputs add half a unit in the last place (at most 2^-8 of the value); a code in E4M3 half a step (2^-4 of the value, 2^-10 absolute), and
one whole step where the value lies within 1e-5 of a rounding boundary.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2401_13920_b200 import block
    return block


def _case(T, H, dt, slots, seed, rows=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0, mean=0.0: torch.randn(*s, generator=g, device="cuda") * std + mean
    s = dict(h=r(T, H, std=2.0).to(dt), y=None, slot=None, inv=None, gate_w=r(T).abs() + 0.05, w_post=r(H, mean=0.7, std=0.3),
             w_pre=r(H, mean=1.0, std=0.3), dh_out=r(T, H).to(dt), dn=r(T, H).to(dt))
    rows = rows or T + T // 3
    if slots:
        slot = torch.randperm(rows, generator=g, device="cuda")[:T].to(torch.int32)
        slot[torch.rand(T, generator=g, device="cuda") < 0.2] = -1
        inv = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
        kept = torch.nonzero(slot >= 0).squeeze(1)
        inv[slot[kept].long()] = kept.to(torch.int32)
        s.update(slot=slot, inv=inv, y=r(rows, H, std=0.3).to(dt))
    else:
        s.update(y=r(T, H, std=0.3).to(dt))
    if T > 2:
        s["y"][0 if s["slot"] is None else max(int(s["slot"][0]), 0)] = 0      # a row of zeros
        s["h"][1] = 0
    return s


def _rows(s):
    y = s["y"].double()
    if s["slot"] is None:
        return y
    return torch.where((s["slot"] >= 0)[:, None], y[s["slot"].clamp_min(0).long()], 0.0)


def _forward64(s, a, eps):
    v = _rows(s) if s["y"] is not None else torch.zeros_like(s["h"], dtype=torch.float64)
    r = (v.pow(2).mean(1) + eps).rsqrt()
    u = v * r[:, None]
    gate = s["gate_w"].double() if s["gate_w"] is not None else torch.ones(len(v), dtype=torch.float64, device="cuda")
    wp = s["w_post"].double() if s["w_post"] is not None else 1.0
    wn = s["w_pre"].double() if s["w_pre"] is not None else 1.0
    hp = a * s["h"].double() + gate[:, None] * wp * u
    q = (hp.pow(2).mean(1) + eps).rsqrt()
    return hp, hp * q[:, None] * wn, u, hp * q[:, None], r, q


def _near(got, want, dt, scale=None):
    """rel 2e-6 of the row's scale plus half an ulp of the output type (2^-8 of a value bounds it)."""
    scale = want.abs().amax(-1, keepdim=True) if scale is None else scale
    tol = 2e-6 * scale + (2.0 ** -8 * want.abs() if dt == torch.bfloat16 else 0.0) + 1e-12
    err = (got.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())


def _near_code(got, want):
    err = (got.double() - want).abs()
    assert (err <= want.abs() * 2.0 ** -4 + 2.0 ** -10 + 1e-5 * want.abs() + 1e-6).all()


SHAPES = [(1, 8), (1, 1), (3, 64), (7, 256), (130, 520), (300, 1024), (17, 5120), (64, 2560), (5, 777), (33, 1001), (9, 4104), (3, 8191),
          (4, 16384), (2, 16392), (2, 40000), (3, 9999), (1, 8193), (1000, 40), (2500, 96), (700, 3), (301, 13), (400, 6), (2001, 77), (350, 5119), (160, 6001),
          (90, 8184)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("T,H", SHAPES)
def test_forward(K, T, H, dt, slots):
    s = _case(T, H, dt, slots, 11 * T + H)
    h_out, n, ck = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.8, EPS, checkpoint=True)
    hp, nn, u, x, r, q = _forward64(s, float(torch.tensor(0.8)), EPS)
    _near(h_out, hp, dt)
    _near(n, nn, dt)
    assert torch.allclose(ck.r_post.double(), r, rtol=2e-6) and torch.allclose(ck.r_pre.double(), q, rtol=2e-6)
    _near_code(ck.u8, u)
    _near_code(ck.x8, x)


def _grad64(s, a, eps, act):
    """The formulas, from normalised rows u, x and reciprocal norms r, q."""
    u, x, r, q = act
    H = u.shape[1]
    wp = s["w_post"].double() if s["w_post"] is not None else torch.ones(H, dtype=torch.float64, device="cuda")
    wn = s["w_pre"].double() if s["w_pre"] is not None else torch.ones(H, dtype=torch.float64, device="cuda")
    gate = s["gate_w"].double()[:, None] if s["gate_w"] is not None else torch.ones(len(u), 1, dtype=torch.float64, device="cuda")
    dn = s["dn"].double() if s["dn"] is not None else torch.zeros_like(u)
    D = s["dh_out"].double() if s["dh_out"] is not None else torch.zeros_like(u)
    gp = dn * wn
    D = D + q[:, None] * (gp - x * (gp * x).mean(1, keepdim=True))
    k = (D * wp * u).sum(1)
    dv = r[:, None] * gate * (D * wp - u * (k / H)[:, None])
    if s["slot"] is not None:
        dy = torch.zeros(len(s["inv"]), H, dtype=torch.float64, device="cuda")
        kept = s["slot"] >= 0
        dy[s["slot"][kept].long()] = dv[kept]
    else:
        dy = dv
    # scales of the terms that the sums are formed from (their differences may be far smaller)
    sD = (s["dh_out"].double().abs() if s["dh_out"] is not None else 0.0) + q[:, None] * (gp.abs() + x.abs() * (gp * x).abs().mean(1, keepdim=True))
    sv = r[:, None] * gate.abs() * (sD * wp.abs() + u.abs() * (sD * wp * u).abs().sum(1, keepdim=True) / H)
    sy = sv
    if s["slot"] is not None:
        sy = torch.zeros_like(dy)
        sy[s["slot"][kept].long()] = sv[kept]
    scale = dict(dh=sD.amax(1, keepdim=True), dy=sy.amax(1, keepdim=True), k=(sD * wp * u).abs().amax(1) * H ** 0.5 + 1e-6, wp=(gate * sD * u).pow(2).sum(0).sqrt() + 1e-6, wn=(dn * x).pow(2).sum(0).sqrt() + 1e-6)
    return a * D, dy, k, (gate * D * u).sum(0), (dn * x).sum(0), scale


@pytest.mark.parametrize("ck", [False, True])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("T,H", SHAPES)
def test_gradient(K, T, H, dt, slots, ck):
    s = _case(T, H, dt, slots, 13 * T + H)
    h_out, _, c = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.8, EPS, checkpoint=ck)
    if ck:
        act = c.u8.double(), c.x8.double(), c.r_post.double(), c.r_pre.double()
    else:
        v, hp = _rows(s), h_out.double()
        r, q = (v.pow(2).mean(1) + EPS).rsqrt(), (hp.pow(2).mean(1) + EPS).rsqrt()
        act = v * r[:, None], hp * q[:, None], r, q
    got = K.block_norm_grad(s["dh_out"], s["dn"], None if ck else h_out, None if ck else s["y"], checkpoint=c, slot=s["slot"], inv=s["inv"],
                            gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], res_scale=0.8, eps=EPS)
    dh, dy, k, dwp, dwn, sc = _grad64(s, float(torch.tensor(0.8)), EPS, act)
    _near(got[0], dh, dt, sc["dh"])
    _near(got[1], dy, dt, sc["dy"])
    _near(got[2], k, torch.float32, sc["k"])
    # column sums: T terms in chains of at most T / 8 adds
    for g, w, z in ((got[3], dwp, sc["wp"]), (got[4], dwn, sc["wn"])):
        assert ((g.double() - w).abs() <= 4e-6 * z * max(1.0, (T / 8) ** 0.5)).all()


@pytest.mark.parametrize("ck", [False, True])
@pytest.mark.parametrize("T,H", [(5, 8192), (40, 8191), (200, 6664), (7, 6657), (3, 8200), (3, 8193)])
def test_gradient_of_long_fp32_rows(K, T, H, ck):
    """Rows of which two do not fit into shared memory."""
    test_gradient(K, T, H, torch.float32, True, ck)


def test_gradient_against_differences(K):
    """Central differences of the kernel's own fp32 forward pass, in random directions of each argument."""
    T, H = 24, 96
    s = _case(T, H, torch.float32, True, 5)
    A, Bq = s["dh_out"].double(), s["dn"].double()

    def value(**kw):
        q = dict(s, **kw)
        h_out, n, _ = K.block_norm(q["h"], q["y"], q["slot"], q["gate_w"], q["w_post"], q["w_pre"], 0.7, EPS)
        return float((A * h_out.double()).sum() + (Bq * n.double()).sum())

    s["h"][1] = 1.0     # the row of zeros has a gradient of order 1/sqrt(eps): its differences say nothing in fp32
    s["y"][max(int(s["slot"][0]), 0)] = 0.5
    h_out, _, _ = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.7, EPS)
    grads = K.block_norm_grad(s["dh_out"], s["dn"], h_out, s["y"], slot=s["slot"], inv=s["inv"], gate_w=s["gate_w"], w_post=s["w_post"],
                              w_pre=s["w_pre"], res_scale=0.7, eps=EPS)
    g = torch.Generator(device="cuda").manual_seed(9)
    for name, grad in zip(("h", "y", "gate_w", "w_post", "w_pre"), grads):
        d = torch.randn(s[name].shape, generator=g, device="cuda")
        step = 2e-3
        num = (value(**{name: s[name] + step * d}) - value(**{name: s[name] - step * d})) / (2 * step)
        ana = float((grad.double() * d.double()).sum())
        # rounding: |value terms| ~ 24*96 of order 1 at 6e-8 each over 2 steps; curvature: step^2
        assert abs(num - ana) <= 2e-3 * (grad.double().norm() * d.double().norm() / d.numel() ** 0.5 + 1.0), (name, num, ana)


def test_parts_that_are_left_out(K):
    """No branch, no next norm, no weights, no gate: each form agrees with the full formulas with the part's neutral value."""
    T, H, dt = 37, 264, torch.float32
    s = _case(T, H, dt, True, 3)
    base = dict(s, gate_w=None, w_post=None, w_pre=None)
    h_out, n, _ = K.block_norm(s["h"], s["y"], s["slot"], eps=EPS)
    hp, nn, *_ = _forward64(base, 1.0, EPS)
    _near(h_out, hp, dt); _near(n, nn, dt)
    h2, n2, c2 = K.block_norm(s["h"], w_pre=s["w_pre"], eps=EPS, want_h=False, checkpoint=True)          # the first norm of a model
    assert h2 is None and c2.u8 is None
    hp, nn, u, x, r, q = _forward64(dict(s, y=None, gate_w=None), 1.0, EPS)
    _near(n2, nn, dt)
    dh, dy, dg, dwp, dwn = K.block_norm_grad(None, s["dn"], h_out=s["h"], w_pre=s["w_pre"], eps=EPS)
    assert dy is None and dg is None and dwp is None
    w = _grad64(dict(s, dh_out=None, slot=None, gate_w=None, w_post=None), 1.0, EPS, (torch.zeros_like(x), x, r, q))
    _near(dh, w[0], dt, w[5]["dh"])
    h3, n3, c3 = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], None, 0.5, EPS, want_n=False, checkpoint=True)   # the last
    assert n3 is None and c3.x8 is None
    _near(h3, _forward64(dict(s, w_pre=None), 0.5, EPS)[0], dt)
    dh, dy, dg, dwp, dwn = K.block_norm_grad(s["dh_out"], None, y=s["y"], slot=s["slot"], inv=s["inv"], gate_w=s["gate_w"],
                                             w_post=s["w_post"], res_scale=0.5, eps=EPS)
    assert dwn is None
    v = _rows(s)
    r = (v.pow(2).mean(1) + EPS).rsqrt()
    w = _grad64(dict(s, dn=None, w_pre=None), 0.5, EPS, (v * r[:, None], torch.zeros_like(v), r, torch.zeros_like(r)))
    _near(dh, w[0], dt, w[5]["dh"]); _near(dy, w[1], dt, w[5]["dy"])


@pytest.mark.parametrize("H", [128, 131])
def test_infinities_and_nan_stay_in_their_rows(K, H):
    T = 9
    s = _case(T, H, torch.bfloat16, False, 4)
    clean = K.block_norm(s["h"], s["y"], None, s["gate_w"], s["w_post"], s["w_pre"], 1.0, EPS, checkpoint=True)
    y, h = s["y"].clone(), s["h"].clone()
    y[3, 5], y[4, 2], h[5, 7], h[6, 0] = float("nan"), float("inf"), float("nan"), float("-inf")
    out = K.block_norm(h, y, None, s["gate_w"], s["w_post"], s["w_pre"], 1.0, EPS, checkpoint=True)
    rest = [0, 1, 2, 7, 8]
    for a, b in ((clean[0], out[0]), (clean[1], out[1]), (clean[2].u8.float(), out[2].u8.float()), (clean[2].x8.float(), out[2].x8.float())):
        assert torch.equal(a[rest], b[rest])
    assert out[1][3].isnan().all() and out[1][5].isnan().all() and out[2].u8[3].float().isnan().all()
    ga = K.block_norm_grad(s["dh_out"], s["dn"], checkpoint=out[2], gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], eps=EPS)
    gb = K.block_norm_grad(s["dh_out"], s["dn"], checkpoint=clean[2], gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], eps=EPS)
    for i in range(3):
        assert torch.equal(ga[i][rest], gb[i][rest])


@pytest.mark.parametrize("H,ck", [(64, False), (64, True), (777, False), (777, True), (10248, False), (10248, True), (10241, False)])
def test_no_eps_keeps_dropped_tokens(K, H, ck):
    """With eps = 0 a token without a row has an infinite reciprocal norm of nothing, which must stay nothing: the bits of
    an eps that no row's mean square notices."""
    s = _case(40, H, torch.float32, True, 5)
    s["y"] += 0.01
    s["h"] += 0.01
    got = []
    for eps in (0.0, 1e-30):
        h_out, n, c = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.5, eps, ck)
        acts = dict(checkpoint=c) if ck else dict(h_out=h_out, y=s["y"])
        grads = K.block_norm_grad(s["dh_out"], s["dn"], slot=s["slot"], inv=s["inv"], gate_w=s["gate_w"], w_post=s["w_post"],
                                  w_pre=s["w_pre"], res_scale=0.5, eps=eps, **acts)
        got.append([h_out, n, *grads] + ([c.u8.view(torch.uint8), c.x8.view(torch.uint8)] if ck else []))
    assert (s["slot"] < 0).any()
    for a, b in zip(*got):
        assert torch.equal(a, b)
        assert not a.float().isnan().any()


def test_unaligned_rows_in_place_and_repeatable(K):
    """Arrays at odd element offsets take the element-wise kernel; h_out may be h, dh may be dh_out; the bits repeat."""
    from paper_2401_13920_b200 import binding as B
    T, H = 50, 512
    s = _case(T, H, torch.bfloat16, True, 6)
    sh, rows = B.Shape(T, H, 1, 1, 1, B.BF16, 0), len(s["inv"])
    h_out, n, _ = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.9, EPS)
    pad = torch.empty(T * H + 1, dtype=torch.bfloat16, device="cuda")
    odd = pad[1:].view(T, H)
    odd.copy_(s["h"])
    n2 = torch.empty_like(s["h"])
    B.locmoe_block_norm(sh, rows, odd, s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.9, EPS, odd, n2)
    hp, nn, *_ = _forward64(s, 0.9, EPS)
    _near(odd, hp, torch.bfloat16); _near(n2, nn, torch.bfloat16)
    kw = dict(slot=s["slot"], inv=s["inv"], gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], res_scale=0.9, eps=EPS)
    one = K.block_norm_grad(s["dh_out"], s["dn"], h_out, s["y"], **kw)
    two = K.block_norm_grad(s["dh_out"], s["dn"], h_out, s["y"], **kw)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    d = s["dh_out"].clone()
    B.locmoe_block_norm_grad(sh, rows, d, s["dn"], h_out, s["y"], dh=d, **kw)
    assert torch.equal(d, one[0])


def test_offsets_beyond_32_bits(K):
    """T * H above 2^31 elements: the last rows of a bf16 stream of 4.3 GB."""
    T, H = 420000, 5120
    h = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    h[-3:] = torch.randn(3, H, device="cuda")
    n = K.block_norm(h, w_pre=None, eps=EPS, want_h=False)[1]
    hp = h[-3:].double()
    _near(n[-3:], hp * (hp.pow(2).mean(1, keepdim=True) + EPS).rsqrt(), torch.bfloat16)
    assert not n[:-3].any()
    dh = K.block_norm_grad(None, h, h_out=n, eps=EPS, want_dw=False)[0]
    x, d = n[-3:].double(), h[-3:].double()
    q = (x.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
    x = x * q
    want = q * (d - x * (d * x).mean(1, keepdim=True))
    _near(dh[-3:], want, torch.bfloat16, d.abs().amax(1, keepdim=True) * 4)


def test_another_stream(K):
    s = _case(200, 1024, torch.bfloat16, True, 8)
    want = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.9, EPS)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = K.block_norm(s["h"], s["y"], s["slot"], s["gate_w"], s["w_post"], s["w_pre"], 0.9, EPS)
    st.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_autograd(K):
    """BlockNorm against torch's own differentiation of the formulas in 64 bits, both forms of the kept activations."""
    T, H = 40, 160
    s = _case(T, H, torch.float32, True, 10)
    s["h"][1] = 1.0
    leaves = [s[k].double().requires_grad_() for k in ("h", "y", "gate_w", "w_post", "w_pre")]
    kept = (s["slot"] >= 0)[:, None]
    v = torch.where(kept, leaves[1][s["slot"].clamp_min(0).long()], 0.0)
    u = v * (v.pow(2).mean(1, keepdim=True) + EPS).rsqrt()
    hp = 0.9 * leaves[0] + leaves[2][:, None] * leaves[3] * u
    n = hp * (hp.pow(2).mean(1, keepdim=True) + EPS).rsqrt() * leaves[4]
    want = torch.autograd.grad([hp, n], leaves, [s["dh_out"].double(), s["dn"].double()])
    for ck, tol in ((False, 2e-6), (True, 0.06)):
        mine = [s[k].clone().requires_grad_() for k in ("h", "y", "gate_w", "w_post", "w_pre")]
        h_out, nn = K.BlockNorm.apply(*mine, s["slot"], s["inv"], 0.9, EPS, ck)
        got = torch.autograd.grad([h_out, nn], mine, [s["dh_out"], s["dn"]])
        for a, b in zip(got, want):
            assert float((a.double() - b).norm()) <= tol * float(b.norm()) * (1 if ck else 4)
        only = torch.autograd.grad([K.BlockNorm.apply(*mine, s["slot"], s["inv"], 0.9, EPS, ck)[0]], mine, [s["dh_out"]], allow_unused=True)
        assert torch.allclose(only[0].double(), 0.9 * s["dh_out"].double(), rtol=1e-6) and not only[4].any()


def test_no_tokens(K):
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    h_out, n, ck = K.block_norm(e, e, checkpoint=True)
    assert h_out.shape == n.shape == (0, 64) and ck.u8.shape == (0, 64)
    dh, dy, dg, dwp, dwn = K.block_norm_grad(e, e, e, e)
    assert dh.shape == dy.shape == (0, 64) and not dwp.any() and not dwn.any()
