"""The operators of language models as far as they need no GPU: sizes, refusals of the C ABI before any launch, and of the calls
on tensors."""
import ctypes

import pytest
import torch

from paper_2208_04187_b200 import binding, build
from paper_2208_04187_b200 import language as lm


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build.build()


@pytest.mark.parametrize("rows, cols", [(1, 1), (1, 32), (7, 33), (8, 128), (128, 256), (129, 257), (300, 1000), (1, 1 << 20), (1 << 20, 40), (2 ** 31 - 513, 3)])
@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_sizes(rows, cols, fmt):
    lo = binding.div_mx_bytes(rows, cols, fmt)
    stages = -(-cols // (128 if fmt == "e4m3" else 256))
    assert lo.codes_bytes == -(-rows // 8) * 8 * stages * 128
    assert lo.scales_bytes == -(-rows // 128) * stages * (512 if fmt == "e4m3" else 1024)
    assert lo.codes_off == 0 and lo.scales_off == lo.codes_bytes and lo.total_bytes == lo.codes_bytes + lo.scales_bytes
    assert lo.closed_form_bytes == rows * -(-cols // 32) * (33 if fmt == "e4m3" else 17)


def test_mx_refusals():
    L, out = binding.lib(), binding.DivMxLayout()
    N, S, P, A, C = binding.DIV_ERR_NULL, binding.DIV_ERR_SHAPE, binding.DIV_ERR_PARAM, binding.DIV_ERR_ALIGN, binding.DIV_ERR_CAPACITY
    assert L.div_mx_bytes(1, 1, 0, None) == N
    for rows, cols in ((0, 1), (1, 0), (-1, 5), (2 ** 31, 1), (1, 2 ** 31), (2 ** 31 - 512, 1)):
        assert L.div_mx_bytes(rows, cols, 0, ctypes.byref(out)) == S
    assert L.div_mx_bytes(1, 1, 2, ctypes.byref(out)) == P
    big = 1 << 30
    q = L.div_mx_quantize
    assert q(None, 4, 32, 32, 0, 0, 256, big, None, 0, None) == N
    assert q(256, 4, 32, 32, 0, 0, None, big, None, 0, None) == N
    assert q(256, 4, 32, 31, 0, 0, 256, big, None, 0, None) == S
    assert q(256, 0, 32, 32, 0, 0, 256, big, None, 0, None) == S
    assert q(256, 4, 32, 32, 3, 0, 256, big, None, 0, None) == P
    assert q(256, 4, 32, 32, 0, -1, 256, big, None, 0, None) == P
    assert q(258, 4, 32, 32, 0, 0, 256, big, None, 0, None) == A
    assert q(257, 4, 32, 32, 1, 0, 256, big, None, 0, None) == A
    assert q(256, 4, 32, 32, 0, 0, 264, big, None, 0, None) == A
    assert q(256, 4, 32, 32, 0, 0, 256, binding.div_mx_bytes(4, 32, "e4m3").total_bytes - 1, None, 0, None) == C
    assert q(256, 4, 32, 32, 0, 0, None, 0, 256, binding.div_mx_bytes(32, 4, "e4m3").total_bytes - 1, None) == C
    d = L.div_mx_dequantize
    assert d(None, big, 4, 32, 0, 256, 0, None) == N and d(256, big, 4, 32, 0, None, 0, None) == N
    assert d(256, big, 4, 0, 0, 256, 0, None) == S and d(256, big, 4, 32, 5, 256, 0, None) == P
    assert d(264, big, 4, 32, 0, 256, 0, None) == A and d(256, big, 4, 32, 0, 254, 0, None) == A
    assert d(256, 100, 4, 32, 0, 256, 0, None) == C
    m = L.div_mx_matmul
    assert m(None, big, 256, big, 4, 4, 32, 0, 256, 4, 0, None) == N
    assert m(256, big, 256, big, 4, 0, 32, 0, 256, 4, 0, None) == S
    assert m(256, big, 256, big, 4, 4, 32, 0, 256, 3, 0, None) == S
    assert m(256, big, 256, big, 4, 4, 32, 2, 256, 4, 0, None) == P
    assert m(256, big, 256, big, 4, 4, 32, 0, 256, 4, 3, None) == P
    assert m(256, big, 264, big, 4, 4, 32, 0, 256, 4, 0, None) == A
    assert m(256, 10, 256, big, 4, 4, 32, 0, 256, 4, 0, None) == C
    assert m(256, big, 256, 10, 4, 4, 32, 0, 256, 4, 0, None) == C


def test_norm_refusals():
    L, N, S, P, A, C = binding.lib(), *(getattr(binding, "DIV_ERR_" + n) for n in ("NULL", "SHAPE", "PARAM", "ALIGN", "CAPACITY"))
    f = L.div_rms_norm_forward
    ok = dict(x=256, xs=64, r=256, rs=64, w=256, wt=0, rows=3, cols=64, t=0, eps=1e-6, h=256, y=256, b=None, cap=0, fmt=0, s=256, st=None)

    def call(**changed):
        return f(*{**ok, **changed}.values())
    assert call(x=None) == N and call(w=None) == N and call(y=None) == N and call(h=None) == N and call(r=None) == N
    assert call(rows=0) == S and call(cols=0) == S and call(xs=63) == S and call(rs=63) == S
    assert call(t=1, wt=2) == P and call(t=3) == P and call(eps=-1.0) == P and call(eps=float("nan")) == P and call(b=256, cap=1 << 20, fmt=7) == P
    assert call(x=254) == A and call(s=254) == A and call(b=264, cap=1 << 20) == A
    assert call(b=256, cap=100) == C
    out = ctypes.c_uint64()
    assert L.div_rms_norm_workspace(0, 4, ctypes.byref(out)) == S and L.div_rms_norm_workspace(4, 4, None) == N
    need = binding.div_rms_norm_workspace(3, 64)
    b = L.div_rms_norm_backward
    ok2 = dict(dy=256, dys=64, dh=256, dhs=64, h=256, hs=64, w=256, wt=0, r=256, rows=3, cols=64, t=0, dx=256, dw=256, ws=256, wb=need, st=None)

    def back(**changed):
        return b(*{**ok2, **changed}.values())
    for name in ("dy", "h", "w", "r", "dx", "ws"):
        assert back(**{name: None}) == N
    assert back(rows=-1) == S and back(dys=1) == S and back(dhs=1) == S and back(hs=1) == S
    assert back(t=9) == P and back(wt=1) == P
    assert back(dx=255) == A and back(ws=264) == A
    assert back(wb=need - 1) == C


def test_logprob_refusals():
    L, N, S, P, A = binding.lib(), *(getattr(binding, "DIV_ERR_" + n) for n in ("NULL", "SHAPE", "PARAM", "ALIGN"))
    ok = dict(x=256, xs=100, rows=3, v=100, t=0, at=256, top=5, lp=256, e=256, s=256, tl=256, ti=256, st=None)

    def call(**changed):
        return L.div_token_logprobs_forward(*{**ok, **changed}.values())
    for name in ("x", "at", "lp", "e", "s", "tl", "ti"):
        assert call(**{name: None}) == N
    assert call(rows=0) == S and call(v=0) == S and call(xs=99) == S and call(v=2 ** 31) == S
    assert call(t=4) == P and call(top=-1) == P and call(top=33) == P and call(v=4, xs=4) == P
    assert call(x=255) == A and call(at=260) == A and call(ti=260) == A
    ok2 = dict(x=256, xs=100, rows=3, v=100, t=0, at=256, s=256, e=256, dl=256, de=256, dx=256, st=None)

    def back(**changed):
        return L.div_token_logprobs_backward(*{**ok2, **changed}.values())
    for name in ("x", "at", "s", "e", "dx"):
        assert back(**{name: None}) == N
    assert back(rows=0) == S and back(xs=9) == S and back(t=-1) == P and back(dx=254) == A and back(dl=258) == A


def test_calls_on_tensors_refuse_what_does_not_fit():
    x, w = torch.zeros(4, 64), torch.zeros(8, 64)
    for call in (lambda: lm.mx_quantize(x), lambda: lm.mx_quantize_both(x), lambda: lm.mx_quantize_columns(x), lambda: lm.mx_linear(x, w),
                 lambda: lm.rms_norm(x, torch.ones(64)), lambda: lm.rms_norm_mx(x, torch.ones(64)), lambda: lm.mx_norm_linear(x, torch.ones(64), w),
                 lambda: lm.token_logprobs(x, torch.zeros(4, dtype=torch.int64))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for call in (lambda: lm.mx_quantize(x, "e5m2"), lambda: lm.mx_linear(x, w, fmt="int8"), lambda: lm.mx_quantize(torch.zeros(4, 0)),
                 lambda: lm.mx_quantize(torch.tensor(1.0)), lambda: lm.mx_quantize([1.0]), lambda: lm.mx_linear(x, torch.zeros(8, 63)),
                 lambda: lm.mx_linear(x, torch.zeros(64)), lambda: lm.mx_matmul(x, w), lambda: lm.rms_norm(x, torch.ones(64), torch.zeros(4, 63)),
                 lambda: lm.token_logprobs(x, torch.zeros(5, dtype=torch.int64)), lambda: lm.token_logprobs(x, None),
                 lambda: lm.mx_quantize_both(torch.zeros(0, 4)), lambda: lm.DivisionLinear(4, 4, fmt="x"),
                 lambda: lm.token_logprobs(torch.zeros(0, 4), torch.zeros(0, dtype=torch.int64), top=5)):
        with pytest.raises((ValueError, TypeError)):
            call()
    blob = torch.empty(0, dtype=torch.uint8)
    a, b = lm.MxTensor(blob, 2, 64, "e4m3"), lm.MxTensor(blob, 2, 64, "e2m1")
    with pytest.raises(ValueError, match="format"):
        lm.mx_matmul(a, b)
    with pytest.raises(ValueError, match="format"):
        lm.mx_matmul(a, lm.MxTensor(blob, 2, 32, "e4m3"))


def test_rows_of_none():
    q = lm.mx_quantize(torch.zeros(0, 64))
    assert q.shape == (0, 64) and q.dequantize().shape == (0, 64) and q.nbytes == 0
    got = lm.token_logprobs(torch.zeros(2, 0, 10), torch.zeros(2, 0, dtype=torch.int64), top=3)
    assert got.logprobs.shape == (2, 0) and got.top_indices.shape == (2, 0, 3) and got.top_indices.dtype == torch.int64
    w = torch.zeros(8, 64, requires_grad=True)
    y = lm.mx_linear(torch.zeros(0, 64, requires_grad=True), w)
    assert y.shape == (0, 8)
    y.sum().backward()
    assert torch.equal(w.grad, torch.zeros_like(w))


def test_layers_are_replaced_with_their_parameters():
    net = torch.nn.Sequential(torch.nn.RMSNorm(16), torch.nn.Linear(16, 8), torch.nn.Sequential(torch.nn.Linear(8, 4, bias=False), torch.nn.LayerNorm(4)))
    kept = list(net.parameters())
    assert lm.to_division_layers(net, "e2m1") is net
    assert [type(m).__name__ for m in net.modules()] == ["Sequential", "DivisionRMSNorm", "DivisionLinear", "Sequential", "DivisionLinear", "LayerNorm"]
    assert all(a is b for a, b in zip(kept, net.parameters())) and net[1].fmt == "e2m1" and net[0].eps == torch.finfo(torch.float32).eps


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_norm_without_an_epsilon_keeps_torchs(dtype):
    """Rows so small that the epsilon decides: what the replaced norm adds gives torch's own output."""
    norm = torch.nn.RMSNorm(64, dtype=dtype)
    x = (0.01 * torch.randn(5, 64, generator=torch.Generator().manual_seed(1))).to(dtype)
    new = lm.to_division_layers(torch.nn.Sequential(norm))[0]
    f = x.double()
    want = f / (f.square().mean(1, keepdim=True) + new.eps).sqrt()
    # torch rounds in 32 bits on its way (a handful of times), then to dtype
    assert ((norm(x).double() - want).abs() <= (torch.finfo(dtype).eps / 2 + 40 * 2.0 ** -24) * want.abs()).all()


def test_a_layer_used_twice_is_replaced_in_both_places():
    class Net(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.a = torch.nn.Linear(4, 4)
            self.b = self.a
            self.inner = torch.nn.Sequential(self.a, torch.nn.RMSNorm(4))
            self.again = self.inner
            self.none = None
            self.register_module("empty", None)
    net = Net()
    w = net.a.weight
    lm.to_division_layers(net)
    assert type(net.a) is lm.DivisionLinear and net.b is net.a and net.inner[0] is net.a and net.again is net.inner
    assert type(net.inner[1]) is lm.DivisionRMSNorm and net.a.weight is w and net.empty is None
    assert not any(type(m) in (torch.nn.Linear, torch.nn.RMSNorm) for m in net.modules())


def test_refusals_of_the_starved_product():
    m = binding.lib().div_debug_mx_matmul_starved
    big = 1 << 30
    for limit in (0, 100_000_001):
        assert m(256, big, 256, big, 4, 4, 32, 0, 256, 4, 0, None, 0, 0, limit) == binding.DIV_ERR_PARAM
    assert m(None, big, 256, big, 4, 4, 32, 0, 256, 4, 0, None, 0, 0, 1) == binding.DIV_ERR_NULL
    assert m(256, big, 256, big, 1, 4, 32, 1, 256, 4, 0, None, 0, 0, 1) == binding.DIV_ERR_PARAM      # one row of 4 bits: nothing is waited for
