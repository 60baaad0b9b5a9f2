"""The calls around the block's kernels on the GPU: streams, memory, and what autograd makes of them."""
import pytest
import torch

from tests.test_block_norm_gpu import EPS, _case
from tests.test_moe_few_gpu import _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2401_13920_b200 import block
    return block


def _flat(out):
    """The tensors of a result, checkpoints among them."""
    parts = [p for o in out for p in (o if isinstance(o, tuple) else (o,))]
    return [p.view(torch.uint8) if p.dtype is torch.float8_e4m3fn else p for p in parts if p is not None]


def _calls(K):
    x, w_in, w_out, eps = _inputs(12, 512, 1024, 8, 1, bias=True)
    s = _case(300, 520, torch.bfloat16, True, 2)
    kw = dict(slot=s["slot"], gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], res_scale=0.9, eps=EPS)
    h_out, _, _ = K.block_norm(s["h"], s["y"], **kw)
    return [lambda **a: K.moe_few(x, w_in, w_out, K=2, eps=eps, **a),
            lambda **a: K.block_norm(s["h"], s["y"], checkpoint=True, **kw, **a),
            lambda **a: K.block_norm_grad(s["dh_out"], s["dn"], h_out, s["y"], inv=s["inv"], **kw, **a)]


@pytest.mark.parametrize("form", ["stream", "handle", "default", "zero"])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_memory_belongs_to_the_given_stream(K, which, form):
    """A call whose `stream` lags behind: what the current stream allocates and fills after the call must be none of the
    memory that the call's kernels have still to use, its private workspace included."""
    call = _calls(K)[which]
    want = _flat(call())
    torch.cuda.synchronize()
    side, given = torch.cuda.Stream(), None
    if form == "stream":
        lag, here, given = side, torch.cuda.current_stream(), side
    elif form == "handle":
        lag, here, given = side, torch.cuda.current_stream(), side.cuda_stream
    else:   # the call goes to the default stream from inside another one
        lag, here, given = torch.cuda.default_stream(), side, torch.cuda.default_stream() if form == "default" else 0
    with torch.cuda.stream(lag):
        torch.cuda._sleep(20_000_000)          # about 10 ms: everything below is queued long before the kernels run
    with torch.cuda.stream(here):
        got = call(stream=given)
        assert torch.cuda.current_stream() == here
        held = []
        for n in (1 << 10, 1 << 14, 1 << 17, 1 << 19, 1 << 21):      # bytes: sizes of the workspaces and the outputs, each pool of the allocator
            for _ in range(12):
                held.append(torch.full((n,), 0xff, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for a, b in zip(_flat(got), want):
        assert torch.equal(a, b)
    assert all(bool((t == 0xff).all()) for t in held)


@pytest.mark.parametrize("which", [0, 1, 2])
def test_outputs_on_another_stream_wait_for_no_one_elses_readers(K, which):
    """Memory that the current stream has just released, with a reader of it still queued there, is not given to a call on
    another stream."""
    call = _calls(K)[which]
    want = _flat(call())
    shapes = [(t.shape, t.dtype) for t in want]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    old = [torch.zeros(*s, dtype=d, device="cuda") for s, d in shapes]
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    copies = [t.clone() for t in old]          # reads that wait behind the sleep
    del old
    got = _flat(call(stream=side))
    torch.cuda.synchronize()
    assert not any(bool(c.any()) for c in copies)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("ck", [False, True])
def test_rows_by_expert(K, ck):
    """The slot buffer as [E][C][H], as a batched product leaves it: the same bits as its rows one after the other, and a
    gradient of its shape."""
    s = _case(100, 264, torch.bfloat16, True, 6, rows=140)
    assert int(s["slot"].max()) >= 7
    y3 = s["y"].view(7, 20, 264)
    kw = dict(gate_w=s["gate_w"], w_post=s["w_post"], w_pre=s["w_pre"], res_scale=0.9, eps=EPS)
    flat, cube = (K.block_norm(s["h"], y, s["slot"], checkpoint=ck, **kw) for y in (s["y"], y3))
    assert all(torch.equal(a, b) for a, b in zip(_flat([o for o in flat if o is not None]), _flat([o for o in cube if o is not None])))
    acts = lambda y: dict(checkpoint=flat[2]) if ck else dict(h_out=flat[0], y=y)
    want = K.block_norm_grad(s["dh_out"], s["dn"], slot=s["slot"], inv=s["inv"], **acts(s["y"]), **kw)
    got = K.block_norm_grad(s["dh_out"], s["dn"], slot=s["slot"], inv=s["inv"], **acts(y3), **kw)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    leaf = y3.clone().requires_grad_()
    h_out, n = K.BlockNorm.apply(s["h"], leaf, s["gate_w"], s["w_post"], s["w_pre"], s["slot"], s["inv"], 0.9, EPS, ck)
    grad, = torch.autograd.grad([h_out, n], [leaf], [s["dh_out"], s["dn"]])
    assert grad.shape == (7, 20, 264) and torch.equal(grad.view(140, 264), want[1])
    with pytest.raises(ValueError, match="inv"):
        out = K.BlockNorm.apply(s["h"], leaf, s["gate_w"], s["w_post"], s["w_pre"], s["slot"], s["inv"][:120], 0.9, EPS, True)
        torch.autograd.grad(out, [leaf], [s["dh_out"], s["dn"]])


@pytest.mark.parametrize("ck", [False, True])
def test_second_derivatives_are_an_error(K, ck):
    """A penalty on a gradient would be taken for a constant: differentiating it raises instead."""
    s = _case(20, 64, torch.float32, True, 7)
    leaves = [s[k].clone().requires_grad_() for k in ("h", "y", "gate_w", "w_post", "w_pre")]
    h_out, n = K.BlockNorm.apply(*leaves, s["slot"], s["inv"], 0.9, EPS, ck)
    first = torch.autograd.grad([h_out.sum() + n.square().sum()], leaves, create_graph=True)
    loss = n.sum() + sum(g.pow(2).sum() for g in first)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        loss.backward()
    h_out, n = K.BlockNorm.apply(*leaves, s["slot"], s["inv"], 0.9, EPS, ck)     # the first ones are as they were
    again = torch.autograd.grad([h_out.sum() + n.square().sum()], leaves)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("T,H,F,E,k", [(3, 512, 8192, 4, 2), (16, 512, 4096, 8, 2), (128, 1024, 1024, 4, 2), (40, 264, 19000, 4, 2)])
def test_slices_are_joined_behind_their_last_store(K, T, H, F, E, k):
    """The last task to arrive adds up slices that other CTAs have stored: the bits of every repetition, with other inputs
    (and so other slices in the same workspace) in between."""
    x, w_in, w_out, eps = _inputs(T, H, F, E, 3, bias=True)
    xs = [x, -x, x.flip(0)]
    want = [K.moe_few(v, w_in, w_out, K=k, eps=eps)[0] for v in xs]
    bad = torch.zeros(3, dtype=torch.int64, device="cuda")
    for i in range(300):
        out = K.moe_few(xs[i % 3], w_in, w_out, K=k, eps=eps)[0]
        bad[i % 3] += (out != want[i % 3]).sum()
    assert bad.tolist() == [0, 0, 0]


def test_weight_of_a_norm_that_is_not_used(K):
    """Only w_pre needs a gradient and n is not used: zeros, with or without a branch."""
    s = _case(30, 72, torch.float32, False, 8)
    for y in (None, s["y"]):
        for ck in (False, True):
            w = s["w_pre"].clone().requires_grad_()
            h_out, n = K.BlockNorm.apply(s["h"], y, None, None, w, None, None, 1.0, EPS, ck)
            h_out.sum().backward()
            assert w.grad.shape == w.shape and not w.grad.any()


@pytest.mark.parametrize("ck", [False, True])
@pytest.mark.parametrize("branch,scale", [(False, 1.0), (False, 0.5), (True, 1.0)])
def test_gradients_without_the_stream(K, branch, scale, ck):
    """BlockNorm without want_h: n and all gradients as with it."""
    s = _case(60, 200, torch.bfloat16, True, 9)
    got = []
    for want_h in (True, False):
        leaves = [s[k].clone().requires_grad_() for k in (("h", "y", "gate_w", "w_post", "w_pre") if branch else ("h", "w_pre"))]
        h, w = leaves[0], leaves[-1]
        y, gate, wp = leaves[1:4] if branch else (None,) * 3
        sl = (s["slot"], s["inv"]) if branch else (None, None)
        h_out, n = K.BlockNorm.apply(h, y, gate, wp, w, *sl, scale, EPS, ck, want_h)
        assert (h_out is None) != want_h
        got.append([n, *torch.autograd.grad([n], leaves, [s["dn"]])])
    assert all(torch.equal(a, b) for a, b in zip(*got))
