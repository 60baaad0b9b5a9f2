"""The few-token layer's intermediate as two bf16 parts: outputs in which the high parts all but cancel, so that what is left
is what the low parts hold.

W_in's rows come in pairs that differ by a bf16 step in every eighth element, W_out has a pair's columns with opposite signs:
out = sum c (v - v'), and v, v' mostly share their high part.  Bounds, per output: v = high + low + rest with |low| <= 2^-8 |v|,
|rest| <= 2^-8 |low| <= 2^-16 |v| (half a unit of 8 significant bits each), the rests taken as independent: six deviations of
2^-16 / sqrt 3 of the terms' root-sum-square; sums are fp32 (1e-6 of the terms' absolute sum, in the second product and, through
the GeLU whose slope is below 1.13, in the first), erfc and the products around it 2^-20 of v; the scores 2e-6 of themselves;
one rounding to bf16 (2^-8 of the value bounds half a unit).
"""
import math

import pytest
import torch

BF = torch.bfloat16


def make(T, H, F, E, seed, device, pairs=192):
    g = torch.Generator(device=device).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=device)
    half = F // 2
    base = (r(E, half, H) * H ** -0.5).to(BF)
    step = torch.where(torch.rand(E, half, H, generator=g, device=device) < 0.5, -1, 1).to(torch.int16)
    step[..., torch.arange(H, device=device) % 8 != 0] = 0
    step[base == 0] = 0
    other = (base.view(torch.int16) + step).view(BF)            # one unit in the last place up or down (in size)
    order = torch.randperm(F, generator=g, device=device)       # where a pair's two columns lie
    w_in, w_out = torch.empty(E, F, H, dtype=BF, device=device), torch.empty(E, H, F, dtype=BF, device=device)
    w_in[:, order[:half]], w_in[:, order[half:]] = base, other
    c = r(E, H, half).to(BF) * (torch.rand(E, H, half, generator=g, device=device) < min(1.0, pairs / half))
    w_out[:, :, order[:half]], w_out[:, :, order[half:]] = c, -c
    return r(T, H).to(BF), w_in, w_out


def intermediate(x, w):
    """GeLU(W_in x) of one expert in 64 bits, and the absolute sum of its terms."""
    a = x.double() @ w.double().t()
    return 0.5 * a * torch.erfc(-a / math.sqrt(2.0)), x.double().abs() @ w.double().abs().t()


def parts(v):
    hi = v.float().to(BF)
    return hi.double(), (v.float() - hi.float()).to(BF).double()


def expected(x, w_in, w_out, idx, w):
    """Outputs in 64 bits for the choices idx and scores w [K][T], and their tolerance."""
    T, H = x.shape
    out, sq, ab, score = (torch.zeros(T, H, dtype=torch.float64, device=x.device) for _ in range(4))
    for c in range(len(idx)):
        for e in idx[c].unique().tolist():
            t = torch.nonzero(idx[c] == e).squeeze(1)
            v, terms = intermediate(x[t], w_in[e])
            f, wo = w[c, t].double()[:, None], w_out[e].double()
            y = f * (v @ wo.t())
            out[t] += y
            score[t] += y.abs()
            sq[t] += f * f * (v.pow(2) @ wo.pow(2).t())
            ab[t] += f * ((2.0 ** -20 * v.abs() + 1e-6 * v.abs() + 1.13e-6 * terms) @ wo.abs().t())
    return out, 6 * 2.0 ** -16 / math.sqrt(3.0) * sq.sqrt() + ab + 2e-6 * score + 2.0 ** -8 * out.abs() + 1e-9


SHAPES = [(8, 64, 1032, 4), (16, 72, 1000, 4), (32, 72, 18952, 4)]


@pytest.mark.parametrize("T,H,F,E", SHAPES)
def test_the_bound_shows_a_wrong_low_part(T, H, F, E):
    """The layer with its low parts as they should be lies within the bound; without them, with another token's, with those
    of other columns or with twice their value every token is beyond it."""
    x, w_in, w_out = make(T, H, F, E, 1, "cpu")
    idx, w = torch.full((1, T), 2), torch.ones(1, T)
    want, tol = expected(x, w_in, w_out, idx, w)
    hi, lo = parts(intermediate(x, w_in[2])[0])
    over = lambda v: ((v @ w_out[2].double().t()).to(BF).double() - want).abs() > tol
    assert not over(hi + lo).any()
    for wrong in (torch.zeros_like(lo), lo.roll(1, 0), lo.roll(8, 1), lo.roll(F // 2, 1), 2 * lo, -lo):
        assert over(hi + wrong).any(1).all()


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2401_13920_b200 import block
    return block


# tokens of a chunk (t.m) at most and beyond half of the tile's rows, for each variant; k that ends inside a stage
CASES = [(1, 64, 1032, 4, 1), (3, 64, 1032, 4, 1), (8, 64, 1032, 4, 1), (4, 64, 520, 4, 2),                    # up to 8 assignments
         (6, 72, 1000, 4, 2), (8, 72, 1000, 4, 2), (9, 72, 1000, 4, 1), (16, 72, 1000, 4, 1), (16, 72, 1000, 4, 2),   # tiles of 16 tokens
         (20, 72, 1000, 4, 1), (24, 72, 1000, 4, 2), (25, 72, 1000, 4, 1), (70, 72, 264, 4, 1), (128, 64, 2048, 4, 2),
         (17, 72, 18952, 4, 1), (32, 72, 18952, 4, 1), (33, 72, 18952, 4, 1), (40, 72, 18952, 4, 1), (48, 72, 18952, 4, 2),   # of 32 tokens
         (49, 72, 18952, 4, 1), (128, 72, 18952, 4, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("spread", [False, True])
@pytest.mark.parametrize("T,H,F,E,k", CASES)
def test_low_parts(K, T, H, F, E, k, spread):
    """All tokens on the same experts, and spread over them."""
    x, w_in, w_out = make(T, H, F, E, T + F + k, "cuda")
    eps = torch.zeros(E, device="cuda")
    if not spread:
        eps[2], eps[1] = 6.0, 3.0
    for weighted in ((True, False) if k == 1 else (True,)):
        out, idx, w = K.moe_few(x, w_in, w_out, K=k, eps=eps, weighted=weighted)
        if not spread:
            assert (idx[0] == 2).all() and (idx[1:] == 1).all()
        want, tol = expected(x, w_in, w_out, idx, w if weighted else torch.ones_like(w))
        err = (out.double() - want).abs()
        assert (err <= tol).all(), float((err / tol).max())
