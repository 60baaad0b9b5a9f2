"""What the calls around the block's kernels refuse before anything is launched, and their ways around what a host may lack
(no GPU needed: tensors are stand-ins, the library's entry points recorders)."""
import pytest
import torch

BF, F32, I32, U8, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


class StandIn:
    """A contiguous tensor as the checks see it, in the memory of device `index`."""
    def __init__(self, numel, dtype, index=0):
        self._n, self.dtype, self._i = numel, dtype, index
        self.is_cuda, self.device = index >= 0, torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    numel = lambda self: self._n
    get_device = lambda self: self._i
    is_contiguous = lambda self: True
    data_ptr = lambda self: 1 << 20


@pytest.fixture
def B(monkeypatch):
    """The binding on a process whose current device is 0; entry points note that they were called and do nothing."""
    from paper_2401_13920_b200 import binding

    class Lib:
        called = []
        def __getattr__(self, name):
            return lambda *a: self.called.append(name) or 0
    lib = Lib()
    lib.called = []
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    return binding


T, H, F, E = 4, 64, 16, 8
FEW = dict(x=(T * H, BF), w_in=(E * F * H, BF), w_out=(E * F * H, BF), idx_k=(2 * T, I32), w_k=(2 * T, F32), out=(T * H, BF),
           ws=(1 << 20, U8), eps=(E, F32))
NORM = dict(h=(T * H, BF), y=(T * H, BF), slot=(T, I32), gate_w=(T, F32), w_post=(H, F32), w_pre=(H, F32), h_out=(T * H, BF),
            n_out=(T * H, BF), u8=(T * H, E4M3), x8=(T * H, E4M3), r_post=(T, F32), r_pre=(T, F32))
GRAD = dict(dh_out=(T * H, BF), dn=(T * H, BF), h_out=(T * H, BF), y=(T * H, BF), u8=(T * H, E4M3), x8=(T * H, E4M3), r_post=(T, F32),
            r_pre=(T, F32), slot=(T, I32), inv=(T, I32), gate_w=(T, F32), w_post=(H, F32), w_pre=(H, F32), dh=(T * H, BF),
            dy=(T * H, BF), dgate=(T, F32), dw_post=(H, F32), dw_pre=(H, F32), ws=(1 << 20, U8))


def _call(B, which, **over):
    args = {k: StandIn(*v) for k, v in dict(few=FEW, norm=NORM, grad=GRAD)[which].items()}
    args.update(over)
    if which == "few":
        return B.locmoe_moe_few(B.make_shape(T, H, E, 1, 1, B.BF16), K=2, F=F, **args)
    shape = B.Shape(T, H, 1, 1, 1, B.BF16, 0)
    return B.locmoe_block_norm(shape, T, **args) if which == "norm" else B.locmoe_block_norm_grad(shape, T, **args)


@pytest.mark.parametrize("which,name", [(w, n) for w, d in (("few", FEW), ("norm", NORM), ("grad", GRAD)) for n in d])
def test_every_tensor_has_to_be_on_the_current_device(B, which, name):
    _call(B, which)
    assert len(B._lib.called) == 1
    spec = dict(few=FEW, norm=NORM, grad=GRAD)[which][name]
    with pytest.raises(ValueError, match=name):
        _call(B, which, **{name: StandIn(*spec, index=1)})
    with pytest.raises(ValueError):
        _call(B, which, **{name: StandIn(*spec, index=-1)})       # host memory
    assert len(B._lib.called) == 1                                 # nothing was launched


def test_no_tensor_is_on_a_device_before_cuda_is_in_use():
    from paper_2401_13920_b200 import binding
    if torch.cuda.is_initialized():
        assert binding._device() == torch.cuda.current_device()
    else:
        assert binding._device() is None
        with pytest.raises(ValueError):
            binding._arg(torch.zeros(4), F32, 4, "x", binding._device())


@pytest.fixture
def K(B, monkeypatch):
    """The allocating calls on host memory, up to the library's entry points: `K.passed` holds the last call's arguments."""
    from paper_2401_13920_b200 import block

    class Passed(dict):
        pass
    seen = Passed()

    def norm(shape, C_alloc, *a, **kw):
        seen.clear(); seen.update(rows=C_alloc, T=shape.T, H=shape.H, wants_h=len(a) > 8 and a[8] is not None, **kw)
    monkeypatch.setattr(block, "_here", lambda t, name: None)
    monkeypatch.setattr(block, "_rows", lambda n, w, dt: torch.zeros(n, w, dtype=dt))
    monkeypatch.setattr(block, "_flat", lambda n, dt: torch.zeros(n, dtype=dt))
    monkeypatch.setattr(block, "_grad_bytes", lambda *a: 64)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "locmoe_block_norm", norm)

    def grad(shape, C_alloc, *a, **kw):
        assert any(kw[k] is not None for k in ("dh", "dy", "dgate", "dw_post", "dw_pre")), "the library refuses a call without outputs"
        norm(shape, C_alloc, *a, **kw)
    monkeypatch.setattr(B, "locmoe_block_norm_grad", grad)
    monkeypatch.setattr(block, "passed", seen, raising=False)
    return block


def _z(*shape, dt=BF):
    return torch.zeros(*shape, dtype=dt)


def test_a_buffer_by_expert_has_all_its_rows(K):
    """Experts' outputs as [E][C][H] or [D][E][C][H]: every row can be named by a slot, not the first E or D alone."""
    for y in (_z(24, 16), _z(3, 8, 16), _z(2, 3, 4, 16)):
        K.block_norm(_z(5, 16), y, _z(5, dt=I32))
        assert K.passed["rows"] == 24 and K.passed["T"] == 5
        inv = _z(24, dt=I32)
        _, dy, *_ = K.block_norm_grad(_z(5, 16), _z(5, 16), _z(5, 16), y, slot=_z(5, dt=I32), inv=inv)
        assert K.passed["rows"] == 24 and dy.shape == (24, 16)
    K.block_norm(_z(5, 16), _z(3, 16), _z(5, dt=I32))                  # fewer rows than tokens
    assert K.passed["rows"] == 3
    K.block_norm(_z(5, 16), _z(7, 16))                                  # without slots rows beyond the tokens' are not read
    K.block_norm_grad(_z(6, 16), _z(6, 16), _z(2, 3, 16), _z(3, 2, 16))


def test_rows_of_another_width_or_number_are_refused(K):
    h, y, s, inv = _z(6, 16), _z(8, 16), _z(6, dt=I32), _z(8, dt=I32)
    for bad in (_z(16, 8), _z(8, 32), _z(8, 16, 1), _z(128), _z(())):
        with pytest.raises(ValueError, match="y: "):
            K.block_norm(h, bad, s)
        with pytest.raises(ValueError, match="y: "):
            K.block_norm(h, bad)
        with pytest.raises(ValueError, match="y: "):
            K.block_norm_grad(h, h, h, bad, slot=s, inv=inv)
    with pytest.raises(ValueError, match="y: "):
        K.block_norm(h, _z(5, 16))                                      # a token without a row
    with pytest.raises(ValueError, match="y: needed"):
        K.block_norm(h, slot=s)
    for rows in (7, 9):                                                 # not the rows that the slots name
        with pytest.raises(ValueError, match="y: "):
            K.block_norm_grad(h, h, h, _z(rows, 16), slot=s, inv=inv)
    with pytest.raises(ValueError, match="y: "):
        K.block_norm_grad(h, h, h, y)                                   # T rows without slots
    for bad in (_z(3, 32), _z(12, 8), _z(7, 16), _z(5, 16), _z(96)):
        with pytest.raises(ValueError, match="dh_out: "):
            K.block_norm_grad(bad, h, h, y, slot=s, inv=inv)
        with pytest.raises(ValueError, match="h_out: "):
            K.block_norm_grad(h, h, bad, y, slot=s, inv=inv)
        code, r = bad.to(E4M3), _z(6, dt=F32)
        good = h.to(E4M3)
        with pytest.raises(ValueError, match="u8: "):
            K.block_norm_grad(h, h, checkpoint=K.Checkpoint(code, good, r, r), slot=s, inv=inv)
        with pytest.raises(ValueError, match="x8: "):
            K.block_norm_grad(h, h, checkpoint=K.Checkpoint(good, code, r, r), slot=s, inv=inv)
    with pytest.raises(ValueError, match="one of them"):
        K.block_norm_grad(None, None, h, h)
    K.block_norm_grad(h, None, None, y, slot=s, inv=inv)                # h_out is not read without dn
    K.block_norm_grad(h, h, h, y, slot=s, inv=inv)


def test_sizes_beyond_32_bits_are_refused(K):
    one = lambda *s: torch.zeros(1, dtype=BF).expand(*s)               # sizes without the memory
    with pytest.raises(ValueError, match="too large"):
        K.block_norm(one(2 ** 32 + 5, 1))
    with pytest.raises(ValueError, match="too large"):
        K.block_norm(_z(5, 1), one(2 ** 32 + 5, 1), _z(5, dt=I32))
    with pytest.raises(ValueError, match="too large"):
        K.block_norm_grad(_z(5, 1), None, y=one(2 ** 32 + 5, 1), slot=_z(5, dt=I32), inv=torch.zeros(1, dtype=I32).expand(2 ** 32 + 5))
    with pytest.raises(ValueError, match="too large"):
        K.moe_few(one(2 ** 32 + 1, 8), one(1, 8, 8), one(1, 8, 8), K=0)
    with pytest.raises(ValueError, match="too large"):
        K.moe_few(one(1, 8), one(1, 2 ** 32 + 8, 8), one(1, 8, 2 ** 32 + 8))


def test_counts_near_the_largest_int_are_refused():
    """The kernels step over tokens and columns in ints: a count within a grid's stride of the largest one would wrap."""
    import ctypes as C
    from paper_2401_13920_b200 import binding as B
    most, P = 0x7fffffff - 0xffff, 1 << 20
    size = C.c_size_t()
    for T, H, rc in ((most + 1, 1, -7), (0x7fffffff, 1, -7), (1, most + 1, -7), (1, 0x7fffffff, -7), (most, 1, -4), (1, most, -4)):
        sh = B.Shape(T, H, 1, 1, 1, B.BF16, 0)
        norm = B.BlockNorm(h=P + 1, h_out=P, eps=1e-6, res_scale=1.0)      # the last check: a misaligned array
        grad = B.BlockNormGrad(dh_out=P + 1, dh=P, eps=1e-6, res_scale=1.0)
        assert B._lib.locmoe_block_norm(C.byref(sh), 1, C.byref(norm), None) == rc
        assert B._lib.locmoe_block_norm_grad(C.byref(sh), 1, C.byref(grad), None, 0, None) == rc
        assert B._lib.locmoe_block_norm_grad_bytes(C.byref(sh), C.byref(size)) == (rc if rc == -7 else 0)


def test_a_gradient_of_nothing_that_is_there(K):
    """Weights that the loss does not reach have a gradient of zero or none, not an error."""
    h, w = _z(6, 16), torch.ones(16, requires_grad=True)
    h_out, n = K.BlockNorm.apply(h, None, None, None, w)
    h_out.float().sum().backward()                                      # n, which alone has w in it, is not used
    assert w.grad.shape == (16,) and not w.grad.any() and "dh" not in K.passed
    gate = torch.ones(6, requires_grad=True)
    h_out, n = K.BlockNorm.apply(h, None, gate, None, None)             # no branch that the gate would be applied to
    n.float().sum().backward()
    assert gate.grad is None or not gate.grad.any()
    assert K.block_norm_grad(h, None, want_dh=False) == (None,) * 5
    K.block_norm_grad(h, h, h, want_dh=False)                           # w_pre's alone
    assert K.passed["dw_pre"].shape == (16,) and K.passed["dh"] is None


def test_a_stream_nobody_asks_for_is_not_written(K):
    """h' of a norm without a branch is h itself: with want_h = False no copy of it is made."""
    h = _z(6, 16).requires_grad_()
    y = _z(6, 16)
    for checkpoint in (False, True):
        for branch, scale, formed in ((None, 1.0, False), (None, 0.5, not checkpoint), (y, 1.0, not checkpoint)):
            h_out, n = K.BlockNorm.apply(h, branch, None, None, None, None, None, scale, 1e-6, checkpoint, False)
            assert h_out is None and K.passed["wants_h"] == formed
            assert K.BlockNorm.apply(h, branch, None, None, None, None, None, scale, 1e-6, checkpoint)[0] is not None


LOST = """
import sys, types, torch
sys.modules["torch._C._dynamo.guards"] = types.ModuleType("guards")       # as of a torch that has moved it
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
from paper_2401_13920_b200 import binding, block
made = []
torch.empty_strided = lambda *a, **k: made.append((a, k)) or torch.zeros(1)
block._rows(3, 5, torch.float32)
assert made == [(((3, 5), (5, 1)), dict(dtype=torch.float32, device="cuda"))], made
torch.cuda.current_device = lambda: 0
torch.cuda.current_stream = lambda device=None: types.SimpleNamespace(cuda_stream=77)
assert binding._stream(None).value == 77 and binding._stream(5).value == 5
print("fine")
"""


def test_a_torch_without_the_short_ways():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    res = subprocess.run([sys.executable, "-c", LOST], cwd=root, capture_output=True, text=True)
    assert res.returncode == 0 and "fine" in res.stdout, res.stderr


def test_a_torch_without_the_short_way_to_its_device():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch
del torch._C._cuda_getDevice
from paper_2401_13920_b200 import binding
assert binding._device() is None and binding._raw_device is torch.cuda.current_device
print("fine")
"""
    res = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert res.returncode == 0 and "fine" in res.stdout, res.stderr


def test_tensors_without_rows_have_to_be_on_the_current_device_too(monkeypatch):
    """A call without rows launches nothing, so the binding never sees its tensors."""
    from paper_2401_13920_b200 import block
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    block._here(StandIn(0, BF, index=0), "x")
    for t in (StandIn(0, BF, index=1), StandIn(0, BF, index=-1), StandIn(8, BF, index=-1)):
        with pytest.raises(ValueError, match="x: on"):
            block._here(t, "x")
