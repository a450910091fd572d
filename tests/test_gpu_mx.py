"""Microscaled matrices on the GPU: quantising equals the 64-bit statement number for number, products keep to what sums in
32 bits allow."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as lo
from paper_2208_04187_b200 import binding, build
from paper_2208_04187_b200 import language as lm

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = ["e4m3", "e2m1"]


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build.build()


def matrix(rows, cols, dtype, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(rows, 1, generator=g))
    x[torch.rand(rows, cols, generator=g) < 0.05] = 0
    return x.to(TYPES[dtype])


def same(got, want):
    np.testing.assert_array_equal(got.cpu().double().numpy() + 0.0, want + 0.0)


SIZES = [(1, 1), (1, 31), (3, 32), (8, 33), (9, 64), (127, 96), (128, 128), (129, 127), (1, 5000), (31, 256), (257, 384), (300, 513)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", SIZES)
def test_quantising_by_rows_and_columns(rows, cols, dtype, fmt):
    x = matrix(rows, cols, dtype, rows * 1000 + cols)
    want, turned = lo.mx_values(x.double().numpy(), fmt), lo.mx_values(x.double().numpy().T, fmt)
    xd = x.cuda()
    a, b = lm.mx_quantize_both(xd, fmt)
    assert a.shape == (rows, cols) and b.shape == (cols, rows)
    same(a.dequantize(torch.float32), want)
    same(b.dequantize(torch.float32), turned)
    same(lm.mx_quantize(xd, fmt).dequantize(torch.bfloat16), want)              # (exact there too)
    same(lm.mx_quantize_columns(xd, fmt).dequantize(torch.float32), turned)
    same(lm.mx_quantize(xd.t(), fmt).dequantize(torch.float32), turned)         # a transposed matrix, read where it is


@pytest.mark.parametrize("fmt", FORMATS)
def test_strides_and_alignment(fmt):
    big = matrix(70, 700, "bf16", 5).cuda()
    for x in (big[:, :640], big[3:, 8:72], big[:, 1:130], big[::2, :128], big[5:6, 3:40], big[:1].expand(4, 700), big.t()[5:300, :33], big.view(70, 7, 100)[:, 2]):
        q = lm.mx_quantize(x, fmt)
        same(q.dequantize(torch.float32), lo.mx_values(x.cpu().double().numpy(), fmt))
        _, c = lm.mx_quantize_both(x, fmt)
        same(c.dequantize(torch.float32), lo.mx_values(x.cpu().double().numpy().T, fmt))
    three = lm.mx_quantize(big.view(7, 10, 700), fmt)
    assert three.shape == (70, 700)


@pytest.mark.parametrize("fmt", FORMATS)
def test_extremes(fmt):
    inf, nan = float("inf"), float("nan")
    x = torch.zeros(12, 64)
    x[0, 3] = inf
    x[1, 40] = nan
    x[2, :] = torch.linspace(-3.4e38, 3.4e38, 64)
    x[3, :32] = 1e-45
    x[4, :] = torch.logspace(-45, 38, 64)
    x[5, :] = 2.0 ** -130
    x[6, :4] = torch.tensor([448.0, 449, -448, 1e-3])
    x[7, :4] = torch.tensor([6.0, 6.0000005, -6, 0.25])
    x[8, :3] = torch.tensor([-inf, inf, nan])
    x[9, :] = -0.0
    x[10, :] = torch.finfo(torch.float32).tiny
    x[11, 32:] = torch.finfo(torch.float32).min
    a, b = lm.mx_quantize_both(x.cuda(), fmt)
    same(a.dequantize(torch.float32), lo.round_to(lo.mx_values(x.double().numpy(), fmt), "f32"))
    same(b.dequantize(torch.float32), lo.round_to(lo.mx_values(x.double().numpy().T, fmt), "f32"))
    for t in ("bf16", "f16"):
        y = x.clamp(-60000, 60000).to(TYPES[t])
        same(lm.mx_quantize(y.cuda(), fmt).dequantize(torch.float32), lo.round_to(lo.mx_values(y.double().numpy(), fmt), "f32"))


def test_rounding_back_to_half_precision():
    x = torch.tensor([[70000.0, 1.0, -1e-9] + [0.0] * 29])
    got = lm.mx_quantize(x.cuda(), "e4m3").dequantize(torch.float16).cpu()
    assert torch.equal(got, torch.from_numpy(lo.mx_values(x.double().numpy(), "e4m3")).half())


def product(a, b):
    """(a b^T, the sum of the magnitudes) in 64 bits."""
    return a @ b.T, np.abs(a) @ np.abs(b).T


def check_product(y, a, b, dtype):
    # a sum of k products in 32 bits, in any order, with additions that may cut off: k steps of 2^-23 of the magnitudes; then one rounding
    want, size = product(a, b)
    half = torch.finfo(TYPES[dtype]).eps / 2
    bound = a.shape[1] * 2.0 ** -23 * size + half * np.abs(want) * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == "f16" else 0)
    got = y.cpu().double().numpy()
    assert got.shape == want.shape and (np.abs(got - want) <= bound).all()


PRODUCTS = [(1, 1, 1), (1, 128, 32), (1, 300, 4096), (2, 129, 96), (15, 256, 160), (16, 100, 512), (17, 640, 1024), (33, 1000, 300), (64, 65, 2050), (65, 64, 64),
            (100, 100, 100), (128, 128, 256), (129, 257, 385), (300, 20, 77), (513, 1, 40), (700, 513, 288), (200, 1100, 8192), (2300, 2200, 200), (5000, 16, 64)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_products(m, n, k, fmt):
    dtype = ("f32", "bf16", "f16")[(m + n + k) % 3]
    a, b = matrix(m, k, "bf16", m, 0.5), matrix(n, k, "f32", n + 1, 0.5)
    y = lm.mx_matmul(lm.mx_quantize(a.cuda(), fmt), lm.mx_quantize(b.cuda(), fmt), TYPES[dtype])
    assert y.dtype == TYPES[dtype]
    check_product(y, lo.mx_values(a.double().numpy(), fmt), lo.mx_values(b.double().numpy(), fmt), dtype)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("m, n", [(5, 200), (200, 300), (3000, 1500)])
def test_a_nan_stays_in_its_row_and_column(m, n, fmt):
    a, b = matrix(m, 320, "f32", 1, 0.5), matrix(n, 320, "f32", 2, 0.5)
    clean = lm.mx_matmul(lm.mx_quantize(a.cuda(), fmt), lm.mx_quantize(b.cuda(), fmt), torch.float32)
    a[3, 100], b[n - 2, 319] = float("nan"), float("-inf")
    y = lm.mx_matmul(lm.mx_quantize(a.cuda(), fmt), lm.mx_quantize(b.cuda(), fmt), torch.float32)
    bad = torch.zeros(m, n, dtype=torch.bool)
    bad[3], bad[:, n - 2] = True, True
    assert torch.equal(y.isnan().cpu(), bad) and torch.equal(y[~bad.cuda()], clean[~bad.cuda()])


def test_scales_of_any_size():
    a, b = torch.ones(3, 64), torch.ones(130, 64)
    a[0] *= 2.0 ** 100
    a[1] *= 2.0 ** -100
    b[0] *= 2.0 ** 20
    b[1] *= 2.0 ** 60
    for fmt in FORMATS:
        y = lm.mx_matmul(lm.mx_quantize(a.cuda(), fmt), lm.mx_quantize(b.cuda(), fmt), torch.float32).cpu()
        assert torch.equal(y, (a.double() @ b.double().t()).float())


def test_out_rows_may_be_apart_and_nothing_else_is_written():
    a, b = matrix(50, 96, "bf16", 3, 0.5), matrix(90, 96, "bf16", 4, 0.5)
    qa, qb = lm.mx_quantize(a.cuda(), "e4m3"), lm.mx_quantize(b.cuda(), "e4m3")
    for m, n, p, q in ((50, 90, qa, qb), (90, 50, qb, qa)):
        out = torch.full((m + 2, 128), 7.0, device="cuda")
        binding.div_mx_matmul(p.blob.data_ptr(), p.blob.numel(), q.blob.data_ptr(), q.blob.numel(), m, n, 96, "e4m3", out[1:].data_ptr(), 128, "f32",
                              binding.current_stream_handle())
        assert torch.equal(out[1:m + 1, :n], lm.mx_matmul(p, q, torch.float32))
        assert (out[0] == 7).all() and (out[m + 1] == 7).all() and (out[:, n:] == 7).all()


def test_results_repeat_and_survive_a_graph_and_another_stream():
    a, b = matrix(3, 4096, "bf16", 8, 0.5).cuda(), matrix(500, 4096, "bf16", 9, 0.5).cuda()
    w = lm.mx_quantize(b, "e2m1")
    want = lm.mx_matmul(lm.mx_quantize(a, "e2m1"), w)
    for _ in range(5):
        assert torch.equal(lm.mx_matmul(lm.mx_quantize(a, "e2m1"), w), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lm.mx_matmul(lm.mx_quantize(a, "e2m1"), w)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lm.mx_matmul(lm.mx_quantize(a, "e2m1"), w)
    a.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want * 2)


def test_a_long_matrix_passes_32_bits():
    rows, cols = 70000, 65536                                   # 4.6e9 numbers
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[rows - 1, cols - 64:] = torch.arange(64, device="cuda")
    x[rows - 300, :32] = 3.0
    q = lm.mx_quantize(x, "e2m1")
    del x
    y = q.dequantize(torch.bfloat16)
    assert float(y[rows - 300, :32].float().sum()) == 96.0
    same(y[rows - 1:, cols - 64:], lo.mx_values(np.arange(64.0)[None], "e2m1"))
    assert int(torch.count_nonzero(y[:rows - 300])) == 0
    one = lm.mx_quantize(torch.ones(1, cols, device="cuda"), "e2m1")
    p = lm.mx_matmul(q, one, torch.float32)
    assert float(p[rows - 1, 0]) == lo.mx_values(np.arange(64.0)[None], "e2m1").sum() and float(p[rows - 300, 0]) == 96.0
    assert int(torch.count_nonzero(p)) == 2


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, n, k", [(3000, 3100, 4096), (2944, 3585, 4100), (4100, 2305, 8000), (2561, 4000, 3850)])
def test_large_products_of_4_bits(m, n, k, dtype):
    """Tiles by pairs of CTAs: odd numbers of blocks, cut blocks, rows of out that begin anywhere.  Sums of these products are exact in 32 bits
    (numbers of one size: every product is a multiple of the smallest, and sums stay below 2^24 of it), so nothing but the rounding is left."""
    g = torch.Generator("cuda").manual_seed(m)
    a = torch.randint(-6, 7, (m, k), generator=g, device="cuda").float()
    b = torch.randint(-6, 7, (n, k), generator=g, device="cuda").float()
    a[:, ::32], b[:, ::32] = 6, 6                                   # every block's scale is 1
    qa, qb = lm.mx_quantize(a, "e2m1"), lm.mx_quantize(b, "e2m1")
    want = qa.dequantize(torch.float32).double() @ qb.dequantize(torch.float32).double().t()
    y = lm.mx_matmul(qa, qb, TYPES[dtype])
    assert torch.equal(y, want.to(TYPES[dtype]))
    assert torch.equal(lm.mx_matmul(qa, qb, TYPES[dtype]), y)


def test_one_token_of_4_bits():
    """The kernel that reads codes itself: NaN blocks, scales far apart, rows of P that end inside a CTA, in every type of out."""
    a, b = torch.ones(1, 300), torch.ones(77, 300)
    a[0, 32:64] *= 2.0 ** 110
    a[0, 64:] = 0
    b[0, 32:64] *= 2.0 ** -120
    b[1, :32] *= 2.0 ** 127 / 64
    b[2, 32:64] *= 2.0 ** 17
    qb = lm.mx_quantize(b.cuda(), "e2m1")
    y = lm.mx_matmul(lm.mx_quantize(a.cuda(), "e2m1"), qb, torch.float32).cpu()
    assert torch.equal(y, (a.double() @ b.double().t()).float())          # (sums whose smaller term is below half a unit of the larger)
    for dtype in TYPES.values():
        z = lm.mx_matmul(lm.mx_quantize(torch.ones(1, 300).cuda(), "e2m1"), lm.mx_quantize(torch.ones(77, 300).cuda(), "e2m1"), dtype)
        assert torch.equal(z, torch.full((1, 77), 300.0, dtype=dtype, device="cuda"))
        assert torch.equal(lm.mx_matmul(lm.mx_quantize(torch.ones(77, 300).cuda(), "e2m1"), lm.mx_quantize(torch.ones(1, 300).cuda(), "e2m1"), dtype), z.t())
    b[5, 299] = float("nan")
    y = lm.mx_matmul(lm.mx_quantize(a.cuda(), "e2m1"), lm.mx_quantize(b.cuda(), "e2m1"), torch.float32).cpu()
    assert y[0, 5].isnan() and int(y.isnan().sum()) == 1
    a[0, 7] = float("inf")
    assert lm.mx_matmul(lm.mx_quantize(a.cuda(), "e2m1"), qb, torch.float32).isnan().all()


def test_nan_in_a_large_product_of_4_bits():
    a, b = torch.ones(3000, 4096, device="cuda"), torch.ones(3100, 4096, device="cuda")
    a[2999, 4095], b[3099, 0], b[128, 2000] = float("nan"), float("inf"), float("nan")
    y = lm.mx_matmul(lm.mx_quantize(a, "e2m1"), lm.mx_quantize(b, "e2m1"), torch.float32)
    bad = torch.zeros(3000, 3100, dtype=torch.bool, device="cuda")
    bad[2999], bad[:, 3099], bad[:, 128] = True, True, True
    assert torch.equal(y.isnan(), bad) and (y[~bad] == 4096).all()


# (m, n, k, format, width of a tile, CTAs of a cluster, the lanes are columns of out, CTAs of the launch); width 512: pairs
STARVED = [(40, 1000, 4096, "e4m3", 64, 8, True, 64), (9, 700, 2000, "e2m1", 16, 4, True, 24), (300, 200, 4096, "e4m3", 128, 8, False, 48),
           (300, 200, 4096, "e2m1", 128, 8, False, 48), (1280, 2304, 700, "e4m3", 128, 1, False, 148), (33, 20000, 300, "e2m1", 64, 1, True, 148),
           (2300, 2200, 1100, "e4m3", 256, 1, False, 148), (2300, 2200, 1100, "e2m1", 256, 1, False, 148), (3000, 3100, 4096, "e2m1", 512, 2, False, 148)]


def starved(qa, qb, m, n, k, fmt, cta, copy):
    out = torch.full((m, n), 7.0, device="cuda")
    st = binding.lib().div_debug_mx_matmul_starved(qa.blob.data_ptr(), qa.blob.numel(), qb.blob.data_ptr(), qb.blob.numel(), m, n, k, binding.MX_FORMATS[fmt],
                                                   out.data_ptr(), n, binding.DIV_F32, binding.current_stream_handle(), cta, copy, 2_000_000)
    assert st == binding.DIV_OK
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("m, n, k, fmt, width, split, swapped, grid", STARVED)
@pytest.mark.parametrize("cta, copy", [(0, 0), (1, 1), (6, 3)])
def test_a_product_whose_wait_cannot_end_returns(m, n, k, fmt, width, split, swapped, grid, cta, copy):
    """Failure detection without a fault: a CTA waits for codes that nobody asks for, its 2 ms limit runs out, it waits for what it has started and
    leaves.  Where a cluster shares a sum, all of that tile is NaN, whatever copies were on their way; the next call finds everything in order."""
    qa, qb = lm.mx_quantize(matrix(m, k, "bf16", 1, 0.5).cuda(), fmt), lm.mx_quantize(matrix(n, k, "bf16", 2, 0.5).cuda(), fmt)
    want = lm.mx_matmul(qa, qb, torch.float32)
    out = starved(qa, qb, m, n, k, fmt, cta, copy)
    run = -(-k // (128 if fmt == "e4m3" else 256)) // split               # stages of a CTA, at least
    if width < 256 and split > 1 and copy < run:
        p = cta // split % -(-(n if swapped else m) // 128) * 128
        part = (out.t() if swapped else out)[p:p + 128]
        s = cta // split // -(-(n if swapped else m) // 128) * width
        assert part[:, s:s + width].isnan().all()
    assert torch.equal(lm.mx_matmul(qa, qb, torch.float32), want)


@pytest.mark.parametrize("m, n, k, fmt, width, split, swapped, grid", STARVED)
@pytest.mark.parametrize("cta, copy", [(0, 0), (1, 1), (5, 2), (6, 7)])
def test_a_wait_that_cannot_end_gives_nan_for_its_part_alone(m, n, k, fmt, width, split, swapped, grid, cta, copy):
    """Failure detection without a fault: a CTA waits for codes that nobody asks for, its 2 ms limit runs out, and whatever this CTA and its cluster have not
    summed by then is NaN, in whole tiles; everything else is as ever."""
    a, b = matrix(m, k, "bf16", 1, 0.5).cuda(), matrix(n, k, "bf16", 2, 0.5).cuda()
    qa, qb = lm.mx_quantize(a, fmt), lm.mx_quantize(b, fmt)
    want = lm.mx_matmul(qa, qb, torch.float32)
    out = starved(qa, qb, m, n, k, fmt, cta, copy)
    high, wide = (256, 256) if width == 512 else (128, width)
    p, s = (n, m) if swapped else (m, n)
    across = -(-p // high)
    tiles, stages = across * -(-s // wide), -(-k // (128 if fmt == "e4m3" else 256))
    unit, together = cta // split, grid // split
    mine = range(unit, tiles, together)
    if width < 256 and split > 1:                                  # a CTA of a cluster has a run of the stages
        stages = stages * (cta % split + 1) // split - stages * (cta % split) // split
    bad = torch.zeros(p, s, dtype=torch.bool, device="cuda")
    if copy < len(mine) * stages:                                  # (else it asks for fewer, and nothing is left out)
        for t in mine[copy // stages:]:
            bad[t % across * high:(t % across + 1) * high, t // across * wide:(t // across + 1) * wide] = True
        assert bad.any()
    if swapped:
        bad = bad.t()
    assert torch.equal(out.isnan(), bad) and torch.equal(out[~bad], want[~bad])
    assert torch.equal(lm.mx_matmul(qa, qb, torch.float32), want)     # the next call finds everything in order


def check_on_the_device(y, a, b, dtype):
    """As check_product, in 64 bits on the GPU."""
    a, b = a.double(), b.double()
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    half = torch.finfo(TYPES[dtype]).eps / 2
    bound = a.shape[1] * 2.0 ** -23 * size + half * want.abs() * (1 + 2.0 ** -10) + (2.0 ** -25 if dtype == "f16" else 0)
    assert y.shape == want.shape and bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("m, n, k, fmt", [(2300, 2200, 1100, "e4m3"), (2561, 4000, 3850, "e4m3"), (4097, 1025, 2050, "e4m3"), (2300, 2200, 1100, "e2m1"),
                                          (777, 5000, 2720, "e2m1"), (2561, 4001, 3840, "e2m1")])
def test_wide_tiles_past_the_first_turn_of_the_ring(m, n, k, fmt):
    """Tiles of 256 columns whose stages go round the ring several times, more than one tile to a CTA; below the sizes that pairs take."""
    dtype = ("f32", "bf16", "f16")[(m + n + k) % 3]
    qa, qb = lm.mx_quantize(matrix(m, k, "bf16", m, 0.5).cuda(), fmt), lm.mx_quantize(matrix(n, k, "bf16", n + 1, 0.5).cuda(), fmt)
    y = lm.mx_matmul(qa, qb, TYPES[dtype])
    check_on_the_device(y, qa.dequantize(torch.float32), qb.dequantize(torch.float32), dtype)
    assert torch.equal(lm.mx_matmul(qa, qb, TYPES[dtype]), y)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_large_linear_layer_and_its_gradients(fmt):
    m, k, n = 2561, 3850, 4000
    x, w, dy = matrix(m, k, "bf16", 1, 0.5).cuda().requires_grad_(), matrix(n, k, "bf16", 2, 0.5).cuda().requires_grad_(), matrix(m, n, "bf16", 3, 0.5).cuda()
    y = lm.mx_linear(x, w, fmt=fmt)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    q = lambda t: lm.mx_quantize(t.detach(), fmt).dequantize(torch.float32)  # noqa: E731
    check_on_the_device(y, q(x), q(w), "bf16")
    check_on_the_device(dx, q(dy), q(w.t()), "bf16")
    check_on_the_device(dw, q(dy.t()), q(x.t()), "bf16")


@pytest.mark.parametrize("fmt", FORMATS)
def test_raw_pointers(fmt):
    x = matrix(40, 300, "f16", 4).cuda()
    rows, cols = lm.mx_quantize_both(x, fmt)
    st = binding.current_stream_handle()
    a, b = (torch.zeros(int(binding.div_mx_bytes(*s, fmt).total_bytes), dtype=torch.uint8, device="cuda") for s in ((40, 300), (300, 40)))
    binding.div_mx_quantize(x.data_ptr(), 40, 300, 300, "f16", fmt, a.data_ptr(), a.numel(), b.data_ptr(), b.numel(), st)
    for blob, q in ((a, rows), (b, cols)):
        out = torch.empty(q.rows, q.cols, device="cuda")
        binding.div_mx_dequantize(blob.data_ptr(), blob.numel(), q.rows, q.cols, fmt, out.data_ptr(), "f32", st)
        assert torch.equal(out, q.dequantize(torch.float32))


@pytest.mark.parametrize("k", [2560, 2561, 3000, 3841])
def test_four_bit_products_on_both_sides_of_the_pairs_border(k):
    """Sums of whole numbers below 2^24: exact, whichever kernel takes them."""
    g = torch.Generator("cuda").manual_seed(k)
    a, b = (torch.randint(-6, 7, (r, k), generator=g, device="cuda").float() for r in (3500, 3300))
    a[:, ::32], b[:, ::32] = 6, 6
    qa, qb = lm.mx_quantize(a, "e2m1"), lm.mx_quantize(b, "e2m1")
    want = qa.dequantize(torch.float32).double() @ qb.dequantize(torch.float32).double().t()
    assert torch.equal(lm.mx_matmul(qa, qb, torch.float32).double(), want)


@pytest.mark.parametrize("n, k", [(512, 8192), (512, 8193), (10240, 1024), (10241, 1024), (4096, 4096), (4097, 4096), (65, 16400)])
def test_one_token_of_4_bits_on_both_sides_of_its_borders(n, k):
    """Sums of whole numbers below 2^24: exact, whichever kernel takes them."""
    g = torch.Generator("cuda").manual_seed(n + k)
    a, b = (torch.randint(-6, 7, (r, k), generator=g, device="cuda").float() for r in (1, n))
    a[:, ::32], b[:, ::32] = 6, 6
    qa, qb = lm.mx_quantize(a, "e2m1"), lm.mx_quantize(b, "e2m1")
    want = qa.dequantize(torch.float32).double() @ qb.dequantize(torch.float32).double().t()
    assert torch.equal(lm.mx_matmul(qa, qb, torch.float32).double(), want)
    assert torch.equal(lm.mx_matmul(qb, qa, torch.float32).double(), want.t())
