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
