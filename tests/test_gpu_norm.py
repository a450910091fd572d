"""The root-mean-square norm on the GPU, its 8- and 4-bit output and its gradients, against the 64-bit statement."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as lo
from paper_2208_04187_b200 import binding, build
from paper_2208_04187_b200 import language as lm

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}      # half of the smallest step


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build.build()


def make(rows, cols, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(TYPES[dtype])


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def depth(cols):
    """Additions that a number of a row goes through: a thread's own (16384 numbers and less are held 32 a thread; longer rows by 512
    threads), the warp's and the CTA's trees."""
    return max(32, -(-cols // 512) + 8) + 10


def within(got, want, bound):
    got = f64(got)
    assert got.shape == np.shape(want) and (np.abs(got - want) <= bound).all(), float(np.max(np.abs(got - want) / bound))


SHAPES = [(1, 1), (2, 7), (1, 64), (5, 65), (3, 255), (4, 256), (9, 768), (1, 4096), (130, 1000), (1100, 520), (2, 4104), (3, 8192), (2, 9001), (2, 16384), (2, 16392),
          (2, 20001)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", SHAPES)
@pytest.mark.parametrize("fused", [False, True])
def test_forward_and_gradients(rows, cols, dtype, fused):
    x, r = make(rows, cols, dtype, rows + cols), make(rows, cols, dtype, rows + cols + 1) if fused else None
    w_type = "f32" if (rows + cols) % 2 else dtype
    w = (1 + 0.3 * make(1, cols, "f32", 3)[0]).to(TYPES[w_type])
    dy, dh = make(rows, cols, dtype, 5), make(rows, cols, dtype, 6) if fused else None
    eps, half, u = 1e-5, torch.finfo(TYPES[dtype]).eps / 2, 2.0 ** -24
    want, h, rstd = lo.rms_norm(f64(x), f64(r), f64(w), eps, dtype)

    xd, wd = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    rd = r.cuda().requires_grad_() if fused else None
    y, hd = lm.rms_norm(xd, wd, rd, eps=eps)
    assert y.dtype == hd.dtype == TYPES[dtype]
    # h is added in 32 bits (exact for the 16-bit types but for one rounding in 2^-24) and rounded
    within(hd, h, half * np.abs(h) * 2.0 ** -10 + (2 * half * np.abs(h) if dtype != "f32" else u * np.abs(h)) + TINY[dtype])
    h = f64(hd)                                                   # what was handed on is what was normalised
    want, _, rstd = lo.rms_norm(h, None, f64(w), eps, dtype)
    d = depth(cols)
    # rstd: half the error of the mean (d additions, products, the division), the root and the division; two products
    slack = (d / 2 + 6) * u
    within(y, want, (half + slack * 1.01) * np.abs(want) + TINY[dtype])

    grads = torch.autograd.grad((y, hd) if fused else y, (xd, rd, wd) if fused else (xd, wd), (dy.cuda(), dh.cuda()) if fused else dy.cuda())
    dx, dw = lo.rms_norm_backward(f64(dy), f64(dh), h, f64(w), rstd)
    n = np.abs(h) * rstd[:, None]
    g = np.abs(f64(dy)) * np.abs(f64(w))
    # every term of dx to slack (n, g, the mean of their products over d additions), then three operations and one rounding
    terms = rstd[:, None] * (g + n * (g * n).mean(1, keepdims=True))
    bound = terms * (4 * slack + (d + 8) * u) + 4 * u * (np.abs(f64(dh)) if fused else 0)
    within(grads[0], dx, bound + half * (np.abs(dx) + bound) + TINY[dtype])
    if fused:
        assert torch.equal(grads[0], grads[1])
    # dw: the rows of a CTA one after another (148 CTAs at least), then the CTAs' sums 32 apart (4 * 8 * 148 at most), then a tree
    size = (np.abs(f64(dy)) * n).sum(0)
    steps = -(-rows // 148) + 8 * 148 * 4 // 32 + 8
    bound = size * (slack + steps * u)
    within(grads[-1], dw, bound + torch.finfo(TYPES[w_type]).eps / 2 * (np.abs(dw) + bound) + TINY[w_type])


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", [(1, 5), (1, 4096), (4, 300), (129, 256), (40, 1000), (1100, 640), (3, 8200), (2, 17000)])
@pytest.mark.parametrize("fused", [False, True])
def test_output_in_few_bits(rows, cols, dtype, fmt, fused):
    x, r = make(rows, cols, dtype, cols), make(rows, cols, dtype, cols + 1) if fused else None
    w = (1 + 0.3 * make(1, cols, "f32", 3)[0]).to(TYPES[dtype])
    q, h = lm.rms_norm_mx(x.cuda(), w.cuda(), None if r is None else r.cuda(), eps=1e-5, fmt=fmt)
    got = f64(q.dequantize(torch.float32))
    want, href, _ = lo.rms_norm(f64(h), None, f64(w), 1e-5, dtype)
    if not fused:
        assert torch.equal(h.cpu(), x)
    slack = (depth(cols) / 2 + 6) * 2.0 ** -24 * 1.01
    # a value within the slack of a border may fall to either side of it; so may the largest one of a block that decides on the scale
    low, high = lo.mx_values(want * (1 - slack), fmt), lo.mx_values(want * (1 + slack), fmt)
    at = lo.mx_values(want, fmt)
    fits = (got == at) | (got == low) | (got == high)
    blocks = np.abs(np.pad(want, ((0, 0), (0, -cols % 32)))).reshape(rows, -1, 32).max(2) / lo.LARGEST[fmt]
    near = np.repeat(np.abs(np.exp2(np.rint(np.log2(np.maximum(blocks, 2.0 ** -126)))) / np.maximum(blocks, 2.0 ** -126) - 1) < 2 * slack, 32, axis=1)[:, :cols]
    assert (fits | near).all()
    assert (got == at).mean() > 0.99
    # the product takes it as it is
    v = make(24, cols, "bf16", 9)
    p = lm.mx_matmul(q, lm.mx_quantize(v.cuda(), fmt), torch.float32)
    ref = got @ lo.mx_values(f64(v), fmt).T
    size = np.abs(got) @ np.abs(lo.mx_values(f64(v), fmt)).T
    within(p, ref, cols * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(ref) + 1e-300)


def test_strides_and_leading_dimensions():
    big = make(60, 300, "bf16", 1).cuda()
    w = torch.ones(256, device="cuda", dtype=torch.bfloat16)
    for x in (big[:, :256], big[:, 3:259], big[::3, 8:264], big[:1, :256].expand(5, 256)):
        y, _ = lm.rms_norm(x, w)
        z, _ = lm.rms_norm(x.contiguous(), w)
        assert torch.equal(y, z)
        y, h = lm.rms_norm(x.contiguous(), w, x)
        z, k = lm.rms_norm(x.contiguous(), w, x.contiguous())
        assert torch.equal(y, z) and torch.equal(h, k)
    x = make(60, 256, "f32", 2).cuda().view(3, 4, 5, 256)
    y, h = lm.rms_norm(x, torch.ones(256, device="cuda"), x)
    assert y.shape == h.shape == x.shape and torch.equal(h, 2 * x)
    x.requires_grad_()
    y, h = lm.rms_norm(x, torch.ones(256, device="cuda"))
    assert h is x
    y.sum().backward()                                            # (a gradient of one number, expanded)
    assert x.grad.shape == x.shape


def test_rows_of_zeros_infinities_and_nan():
    x = torch.zeros(4, 128)
    x[1, 3], x[2, 5] = float("inf"), float("nan")
    x[3] = 1
    y, _ = lm.rms_norm(x.cuda(), torch.ones(128, device="cuda"), eps=1e-6)
    assert (y[0] == 0).all() and y[1, 3].isnan() and y[2].isnan().all() and torch.allclose(y[3], torch.ones(128, device="cuda"), atol=1e-5)
    q, _ = lm.rms_norm_mx(x.cuda(), torch.ones(128, device="cuda"), eps=1e-6)
    d = q.dequantize(torch.float32)
    assert (d[0] == 0).all() and d[1, :32].isnan().all() and d[2].isnan().all() and (d[3] == 1).all()


def test_only_what_is_wanted_is_computed():
    x, r, w = (make(6, 96, "f32", i).cuda().requires_grad_() for i in range(3))
    w = torch.ones(96, device="cuda")
    y, h = lm.rms_norm(x, w, r)
    (g,) = torch.autograd.grad(h, x, torch.ones_like(h), retain_graph=True)      # y takes no part
    assert torch.equal(g, torch.ones_like(h))
    g1, g2 = torch.autograd.grad(y, (x, r), torch.ones_like(y))
    assert torch.equal(g1, g2)
    with pytest.raises(ValueError, match="weight"):
        lm.rms_norm(x, torch.ones(95, device="cuda"))
    with pytest.raises(ValueError, match="residual"):
        lm.rms_norm(x, w, r.detach().half())
    with pytest.raises(ValueError, match="weight"):
        lm.rms_norm(x.detach().half(), torch.ones(96, device="cuda", dtype=torch.bfloat16))


def test_rows_behind_the_last_are_left_alone():
    x, w = make(3, 104, "bf16", 1).cuda(), torch.ones(104, device="cuda", dtype=torch.bfloat16)
    out = torch.full((5, 104), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.div_rms_norm_forward(x.data_ptr(), 104, None, 0, w.data_ptr(), "bf16", 3, 104, "bf16", 1e-6, None, out[1:].data_ptr(), None, 0, "e4m3", None,
                                 binding.current_stream_handle())
    assert (out[0] == 7).all() and (out[4] == 7).all() and torch.equal(out[1:4], lm.rms_norm(x, w)[0])


# more rows than groups of threads, and no multiple of them: every size of group, aligned rows and others
MANY = [(10007, 100, "bf16"), (10007, 104, "f32"), (3001, 520, "f16"), (3001, 521, "bf16"), (1000, 4096, "bf16"), (2500, 4096, "f32"), (1501, 2600, "bf16"),
        (1501, 2601, "f16"), (701, 5000, "f16"), (701, 4999, "f32"), (500, 8192, "bf16"), (500, 8190, "bf16"), (900, 9001, "bf16"), (700, 16392, "f16")]


@pytest.mark.parametrize("rows, cols, dtype", MANY)
@pytest.mark.parametrize("fused", [False, True])
def test_gradients_of_many_rows(rows, cols, dtype, fused):
    """A group of threads goes from row to row: the next row's reads on their way, the weight's sums carried on, the long rows' in memory."""
    groups = binding.div_rms_norm_workspace(rows, cols) // (4 * cols)
    assert rows > groups and rows % groups
    test_forward_and_gradients(rows, cols, dtype, fused)


@pytest.mark.parametrize("dtype", TYPES)
def test_raw_pointers_backward(dtype):
    rows, cols = 40, 264
    dy, dh, x = (make(rows, cols, dtype, i).cuda() for i in range(3))
    w = (1 + 0.3 * make(1, cols, "f32", 3)[0]).to(TYPES[dtype]).cuda()
    a, r, v = x.clone().requires_grad_(), torch.zeros_like(x).requires_grad_(), w.clone().requires_grad_()
    y, h = lm.rms_norm(a, v, r, eps=1e-5)
    want = torch.autograd.grad((y, h), (a, v), (dy, dh))
    st, p = binding.current_stream_handle(), torch.Tensor.data_ptr
    out, hh, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    binding.div_rms_norm_forward(p(x), cols, p(r), cols, p(w), dtype, rows, cols, dtype, 1e-5, p(hh), p(out), None, 0, "e4m3", p(rstd), st)
    assert torch.equal(out, y) and torch.equal(hh, h)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(binding.div_rms_norm_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    binding.div_rms_norm_backward(p(dy), cols, p(dh), cols, p(hh), cols, p(w), dtype, p(rstd), rows, cols, dtype, p(dx), p(dw), p(ws), ws.numel(), st)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
