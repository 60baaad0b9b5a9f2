"""Values that the other tests of the sorted-token operators do not reach: the balance loss's gradient by itself, group means that are
not numbers, the activations far from zero.  A rounding to bf16 is off by 2^-8 of the value at most, to fp32 by 2^-24."""
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,H,E,K", [(2, 64, 4, 1), (50, 64, 8, 2), (301, 120, 5, 3), (2000, 512, 32, 1)])
def test_the_balance_loss_and_its_gradient_alone(X, T, H, E, K, dt):
    """weight * alpha * E * sum_i f_i P_i against 64 bits, f of the kernel's own first choices, some experts liked more; and that a
    loss with any of its factors lost or its sign turned would be seen."""
    g, alpha, weight = gen(T), 0.07, 2.5
    n = H // E
    like = (torch.linspace(0.0, 1.0, E, device="cuda") + 0.1)[None, :, None]
    x = (randn(g, T, E, n) + like).reshape(T, H).to(dt).requires_grad_()
    eps = randn(g, E, std=0.05).requires_grad_()
    _, _, aux, idx, *_ = X.RouteSort.apply(x, eps, E, K, alpha)
    (weight * aux).backward()
    f = torch.bincount(idx[0].long(), minlength=E).double() / T
    G = x.detach().double().view(T, E, n).mean(2) + eps.detach().double()
    p = torch.softmax(G.clamp_min(0.0), 1)
    want = alpha * E * float((f * p.mean(0)).sum())
    # the loss: sums of T and E terms in fp32, the exponentials a few steps
    assert abs(float(aux.detach()) - want) <= (T + E + 16) * 2.0 ** -24 * want + 1e-5 * want
    q = weight * alpha * E / T * f                              # gradient of every token's p
    m = (p * q).sum(1, keepdim=True)
    dG = torch.where(G > 0, p * (q - m), 0.0)
    # as in the router's other test: G is off by `off`, p by 2 off, the exponential, the sum and the division; q by 8 roundings
    off = (n + 3) * 2.0 ** -24 * (x.detach().double().abs().view(T, E, n).mean(2) + eps.detach().double().abs())
    clear = G.abs() > off
    assert clear.double().mean() > 0.99
    rel = 2 * off.amax(1, keepdim=True) + (E + 8) * 2.0 ** -24
    tol = p * (q + m) * (2 * rel + (E + 13) * 2.0 ** -24)
    spread = lambda a: (a / n)[:, :, None].expand(T, E, n).reshape(T, H)
    sure = spread(clear.double() * n) > 0.5

    def fits(scale):
        dx, deps = spread(dG) * scale, dG.sum(0) * scale
        a = (x.grad.double() - dx).abs() <= HALF[dt] * dx.abs() + (1 + HALF[dt]) * spread(tol) * abs(scale)
        b = (eps.grad.double() - deps).abs() <= abs(scale) * ((tol + torch.where(clear, 0.0, p * (q + m))).sum(0) + (T + 2) * 2.0 ** -24 * dG.abs().sum(0))
        return bool((a | ~sure).all()), bool(b.all())
    assert fits(1.0) == (True, True)
    for scale in (1 / E, T, 1 / alpha, 1 / weight, -1.0, 0.0):
        assert fits(scale) == (False, False)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,K,H,E", [(9, 2, 2560, 32), (33, 3, 777, 21), (50, 8, 1024, 1024), (31, 3, 1236, 6), (7001, 1, 72, 8), (6500, 2, 256, 64)])
def test_a_group_mean_that_is_no_number_counts_as_zero(X, T, K, H, E, dt):
    """As in the forward pass: the same choices, scores and gradients, bit for bit, as for a group whose ReLU gives nothing."""
    g, n = gen(T), H // E
    x = randn(g, T, H, dtype=dt)
    hit = torch.rand(T, E, generator=g, device="cuda") < 0.2
    one = hit[:, :, None] & (torch.arange(n, device="cuda") == torch.randint(0, n, (T, E, 1), generator=g, device="cuda"))
    nan = torch.where(one, float("nan"), x.view(T, E, n).float()).to(dt).reshape(T, H)
    none = torch.where(hit[:, :, None], -1.0, x.view(T, E, n).float()).to(dt).reshape(T, H)
    eps = randn(g, E, std=0.1)
    dxs, dw, dp = randn(g, K * T, H, dtype=dt), randn(g, K, T), randn(g, E)
    got = []
    for v in (nan, none):
        _, w_k, _, idx, offsets, slot, inv = X.RouteSort.apply(v, eps, E, K, 0.0)
        order = X.Order(offsets, slot, inv)
        got.append([w_k, idx, *X.sort_rows_grad(dxs, order, v, idx, dw, eps, dp), *X.sort_rows_grad(None, order, v, idx, dw, eps, dp)])
    for a, b in zip(*got):
        assert bool(b.isfinite().all()) and torch.equal(a, b)


def every_bf16(limit):
    z = torch.arange(-2 ** 15, 2 ** 15, device="cuda", dtype=I32).to(torch.int16).view(BF)
    z = z[z.isfinite() & (z.abs() <= limit)]
    return torch.cat([z, z[:-z.numel() % 64]]).view(-1, 64).contiguous()


def phi64(v):
    return torch.special.erfc(-v / math.sqrt(2.0)) / 2                  # keeps its digits below zero


@pytest.mark.parametrize("few", [False, True])
def test_gelu_keeps_its_digits_far_below_zero(X, few):
    """Every bf16 number of [-12, 12] through an expert that is the identity: relative to the value, also where that is small."""
    z = every_bf16(12.0)
    w = torch.eye(64, dtype=BF, device="cuda")[None].contiguous()
    v = z.double()
    want, slope = v * phi64(v), phi64(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    # erfc by its own fit: 1e-6 of the value.  The exponential's argument is rounded three times and as large as z^2 / 2 log2(e), the
    # function itself and the reciprocal are a few steps each.
    rel = 1e-6 + (3 * v * v / 2 + 24) * 2.0 ** -24
    step = 4 if few else z.shape[0]
    for a in range(0, z.shape[0], step):
        rows = z[a:a + step].contiguous()
        offsets = torch.tensor([0, rows.shape[0]], dtype=I32, device="cuda")
        y, kept = X.expert_linear(rows, w, offsets, act="gelu", want_z=True)
        s = slice(a, a + step)
        assert torch.equal(kept, rows)
        tiny = 2.0 ** -126                                              # what is below the normal numbers may be zero
        assert ((y.double() - want[s]).abs() <= (2.0 ** -8 + 1.01 * rel[s]) * want[s].abs() + tiny).all()
        if few:
            continue
        one = torch.ones_like(rows)                                     # dx = 1 * slope(z), the identity being its own transpose
        dx, _, _ = X.expert_linear_grad(one, None, w, offsets, rows, "gelu", want_dw=False)
        # next to its zero the slope is the difference of two terms
        size = phi64(v) + v.abs() * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        assert ((dx.double() - slope).abs() <= 2.0 ** -8 * slope.abs() + 1.01 * rel * size + tiny).all()
