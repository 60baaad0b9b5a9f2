"""The example's dropless training step, and a whole step captured into a graph, against autograd in 64 bits."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import moe_block
    finally:
        sys.path.pop(0)
    return moe_block


def inputs(T, H, F, E, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0, mean=0.0, dt=torch.float32: (torch.randn(*s, generator=g, device="cuda") * std + mean).to(dt)
    return r(T, H, dt=BF), [r(H, std=0.1, mean=1.0), r(E, F, H, std=0.1, dt=BF), r(E, H, F, std=0.1, dt=BF), r(H, std=0.1, mean=0.5), r(H, std=0.1, mean=1.0)], \
        r(T, H)


def step64(X, h, params, target, K, alpha):
    """The loss in 64 bits; the choices are those of the bf16 router, taken from its input as the norm rounds it."""
    from paper_2401_13920_b200 import block, experts
    E = params[1].shape[0]
    n_bf = block.block_norm(h, w_pre=params[0], eps=X.EPS, want_h=False)[1]
    idx = experts.RouteSort.apply(n_bf, None, E, K, 0.0)[3].long()
    w_pre, w_in, w_out, w_post, w_next = leaves = [p.double().requires_grad_() for p in params]
    norm = lambda v: v * (v.pow(2).mean(1, keepdim=True) + X.EPS).rsqrt()
    x = h.double()
    n = norm(x) * w_pre
    p = torch.softmax(n.view(n.shape[0], E, -1).mean(2).clamp_min(0.0), 1)
    y = 0.0
    for k in range(K):
        a = torch.einsum("th,tfh->tf", n, w_in[idx[k]])
        y = y + p.gather(1, idx[k][:, None]) * torch.einsum("tf,thf->th", a * torch.special.ndtr(a), w_out[idx[k]])
    f = torch.bincount(idx[0], minlength=E).double() / n.shape[0]
    loss = (norm(x + w_post * norm(y)) * w_next - target.double()).square().mean() + alpha * E * (f * p.mean(0)).sum()
    loss.backward()
    return loss.detach(), [l.grad for l in leaves]


@pytest.mark.parametrize("T,H,F,E,K", [(200, 64, 128, 4, 2), (77, 128, 72, 8, 1), (9, 96, 264, 3, 3)])
def test_dropless_training_step(X, T, H, F, E, K):
    h, params, target = inputs(T, H, F, E, T)
    leaves = [p.clone().requires_grad_() for p in params]
    loss = X.train_step_dropless(h, *leaves, target, K=K)
    want, grads = step64(X, h, params, target, K, 0.01)
    # bf16 roundings of the rows, the activation, their gradients and the outputs (2^-8 of an element each at most) and the norms'
    # 8-bit checkpoints (2^-4 of an element at most, 2^-4 / sqrt(3) in the mean, once for each of the two norms' gradients)
    assert abs(float(loss) - float(want)) <= 4 * 2.0 ** -8 * float(want)
    for leaf, g in zip(leaves, grads):
        assert float((leaf.grad.double() - g).norm()) <= (2 * 2.0 ** -4 / 3 ** 0.5 + 8 * 2.0 ** -8) * float(g.norm())


def test_a_captured_training_step(X):
    """Forward and backward of the layer in one graph, replayed on other inputs."""
    from paper_2401_13920_b200 import experts
    T, H, F, E, K = 150, 64, 136, 4, 2
    _, params, _ = inputs(T, H, F, E, 1)
    x = torch.zeros(T, H, dtype=BF, device="cuda")
    w_in, w_out = (p.clone().requires_grad_() for p in params[1:3])
    xl = x.clone().requires_grad_()

    def run():
        for t in (xl, w_in, w_out):
            t.grad = None
        out, aux = experts.moe_layer(xl, w_in, w_out, K, alpha=0.1)
        (out.float().square().sum() + aux).backward()
        return out.detach()
    with torch.no_grad():
        xl.copy_(inputs(T, H, F, E, 2)[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    for t in (xl, w_in, w_out):
        t.grad = None
    with torch.cuda.graph(graph):
        out = run()
    got_at = [xl.grad, w_in.grad, w_out.grad]
    for seed in (3, 4):
        with torch.no_grad():
            xl.copy_(inputs(T, H, F, E, seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone()] + [t.clone() for t in got_at]
        fresh = [t.detach().clone().requires_grad_() for t in (xl, w_in, w_out)]
        o, aux = experts.moe_layer(*fresh, K, alpha=0.1)
        (o.float().square().sum() + aux).backward()
        for a, b in zip(got, [o.detach()] + [t.grad for t in fresh]):
            assert torch.equal(a, b)


CHILD = """
import torch
from paper_2401_13920_b200 import experts
BF = torch.bfloat16
x = torch.randn(40, 64, device="cuda").to(BF).requires_grad_()
w_in, w_out = (torch.randn(4, *s, device="cuda").to(BF).requires_grad_() for s in ((72, 64), (64, 72)))
leaves = (x, w_in, w_out)
def run():
    return experts.moe_layer(*leaves, 2, residual=x if RESIDUAL else None)[0].float().square().sum()
s = torch.cuda.Stream()
with torch.cuda.stream(s):
    run().backward()
torch.cuda.synchronize()
for live in (True, False):
    for t in leaves:
        t.grad = None
    eager = run() if live else None
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph):
            run().backward()
        print("captured")
        graph.replay()
        for t, g in zip(leaves, torch.autograd.grad(run(), leaves)):
            assert torch.equal(t.grad, g)
    except RuntimeError as e:
        print("refused" if "a captured backward pass" in str(e) else e)
    torch.cuda.synchronize()
"""


@pytest.mark.parametrize("residual", [False, True])
def test_a_captured_backward_pass_refuses_a_graph_on_the_default_stream(residual):
    """In a process of its own, which has to live on and capture the step once the other graph is gone."""
    done = subprocess.run([sys.executable, "-c", CHILD.replace("RESIDUAL", str(residual))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    assert done.stdout.split() == ["refused", "captured"], done.stdout


def test_example_main_runs(X, capsys):
    X.main()
    assert "without a capacity" in capsys.readouterr().out
