"""Log probabilities, entropies, alternatives and their gradient on the GPU against the 64-bit statement."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as lo
from paper_2208_04187_b200 import binding, build
from paper_2208_04187_b200 import language as lm

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build.build()


def make(rows, vocab, dtype, seed, scale=3.0, masked=0.0):
    g = torch.Generator().manual_seed(seed)
    x = scale * torch.randn(rows, vocab, generator=g)
    x[torch.rand(rows, vocab, generator=g) < masked] = -INF
    t = torch.randint(0, vocab, (rows,), generator=g)
    x.scatter_(1, t[:, None], torch.randn(rows, 1, generator=g))
    return x.to(TYPES[dtype]), t


def f64(t):
    return t.detach().cpu().double().numpy()


def slack(x):
    """What a row's log s and t / s may be off by: the exponential's 2 units (2^-22) and its argument, rounded twice and times log2 e; a
    thread's additions, trees over the CTA and the cluster, rescalings."""
    with np.errstate(all="ignore"):
        m = x.max(1)
        a = x - np.where(np.isfinite(m), m, 0)[:, None]
        e = np.exp(a)
        mean = np.where(e > 0, -a * e, 0).sum(1) / np.maximum(e.sum(1), 1e-300)
    steps = -(-x.shape[1] // 256) + 40
    return (steps + 8 * mean + 8) * 2.0 ** -24 + 2.0 ** -21, mean


def check(x, t, top, got):
    lp, ent, tv, ti = lo.token_logprobs(f64(x), t.numpy(), top)
    off, mean = slack(f64(x))
    u = 2.0 ** -23
    for value, want, bound in ((got.logprobs, lp, off + u * (np.abs(lp) + 20)), (got.entropy, ent, off * (2 + 2 * mean) + u * (ent + 20)),
                               (got.top_logprobs, tv, off[:, None] + u * (np.abs(tv) + 20))):
        v = f64(value)
        assert value.dtype == torch.float32 and v.shape == want.shape
        fin = np.isfinite(want)
        assert np.array_equal(v[~fin], want[~fin], equal_nan=True)
        assert (np.abs(v - want)[fin] <= np.broadcast_to(bound, want.shape)[fin]).all()
    assert np.array_equal(got.top_indices.cpu().numpy(), ti)


SHAPES = [(1, 1), (1, 2), (3, 7), (5, 100), (2, 255), (40, 1000), (300, 513), (1, 4097), (7, 20011), (1, 131072), (3, 65537), (600, 2049)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab", SHAPES)
def test_forward(rows, vocab, dtype):
    x, t = make(rows, vocab, dtype, rows + vocab, masked=0.3 if vocab > 50 else 0.0)
    for top in sorted({0, 1, min(5, vocab), min(20, vocab), min(32, vocab)}):
        check(x, t, top, lm.token_logprobs(x.cuda(), t.cuda(), top=top))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, vocab", SHAPES)
def test_gradient(rows, vocab, dtype):
    x, t = make(rows, vocab, dtype, rows * vocab, masked=0.2 if vocab > 50 else 0.0)
    g = torch.Generator().manual_seed(1)
    dl, de = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    t[::3] = torch.where(torch.arange(0, rows, 3) % 2 == 1, -1, t[::3])                  # some rows without a token
    xd = x.cuda().requires_grad_()
    lp, ent = lm.token_logprobs(xd, t.cuda())[:2]
    off, _ = slack(f64(x))
    half = torch.finfo(TYPES[dtype]).eps / 2
    for pair in ((dl, de), (dl, None), (None, de)):
        outs = [(o, d.cuda()) for o, d in zip((lp, ent), pair) if d is not None]
        (got,) = torch.autograd.grad([o for o, _ in outs], xd, [d for _, d in outs], retain_graph=True)
        a, b = (np.zeros(rows) if d is None else f64(d) for d in pair)
        want = lo.token_logprobs_backward(f64(x), t.numpy(), a, b)
        with np.errstate(all="ignore"):
            xs = f64(x)
            logp = xs - xs.max(1, keepdims=True)
            logp = logp - np.log(np.exp(logp).sum(1, keepdims=True))
            p = np.exp(logp)
            size = np.where(p > 0, p * (np.abs(a)[:, None] + np.abs(b)[:, None] * (np.abs(logp) + f64(ent)[:, None])), 0)
            # p: log p to off and two roundings of x - m; then a few operations
            rel = off[:, None] * 2 + (3 * np.where(p > 0, np.abs(logp) + 20, 0) + 8) * 2.0 ** -24 + 2.0 ** -21
            entropy = np.where(p > 0, p, 0) * (np.abs(b) * (off * (2 + 2 * slack(xs)[1]) + 2.0 ** -22 * (f64(ent) + 20)))[:, None]
        bound = size * rel + entropy + 2.0 ** -23 * np.abs(a)[:, None]
        bound = bound + half * (np.abs(want) + bound) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -126)
        assert got.dtype == TYPES[dtype] and (np.abs(f64(got) - want) <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 1000, 30001])
def test_what_masks_leave(vocab, dtype):
    least = torch.finfo(TYPES[dtype]).min
    x, t = make(12, vocab, dtype, vocab)
    x[0] = -INF                                     # nothing
    x[1] = least                                    # the type's lowest value everywhere: a uniform distribution
    x[2] = -INF
    x[2, 7] = 1.5                                   # one token
    x[3] = least
    x[3, vocab - 1] = 0.25
    x[4, 3] = NAN
    x[5, 5] = INF
    x[6] = 2.0                                      # all equal
    x[7] = -torch.arange(vocab).to(x.dtype)         # sorted, either way
    x[8] = torch.arange(vocab).to(x.dtype) / vocab
    x[9] = 0.0
    x[9, ::2] = -0.0
    x[10] = NAN
    x[11, :] = least
    x[11, 1:3] = -INF
    t[:] = torch.tensor([0, 5, 7, vocab - 1, 1, 1, 3, 2, vocab - 1, 9, 0, 4])
    for top in (0, 1, 5, 32):
        check(x, t, top, lm.token_logprobs(x.cuda(), t.cuda(), top=top))
    xd = x.cuda().requires_grad_()
    lp, ent = lm.token_logprobs(xd, t.cuda())[:2]
    (g,) = torch.autograd.grad((lp, ent), xd, (torch.ones_like(lp), torch.ones_like(ent)))
    assert (g[0] == 0).all() and g[4].isnan().all() and g[10].isnan().all()
    assert (g[2].abs() < 1e-6).all()
    want = lo.token_logprobs_backward(f64(x)[[1, 3, 6, 7, 8, 9, 11]], t.numpy()[[1, 3, 6, 7, 8, 9, 11]], np.ones(7), np.ones(7))
    np.testing.assert_allclose(f64(g)[[1, 3, 6, 7, 8, 9, 11]], want, rtol=2.0 ** -7, atol=2e-5)


def test_targets_that_are_none_or_outside():
    x, t = make(5, 333, "f32", 1)
    t[1], t[2], t[3] = -100, 333, 2 ** 40
    xd = x.cuda().requires_grad_()
    got = lm.token_logprobs(xd, t.cuda())
    assert got.logprobs[1] == 0 and got.logprobs[2].isnan() and got.logprobs[3].isnan() and got.logprobs[[0, 4]].isfinite().all()
    g = torch.autograd.grad(got.logprobs.sum(), xd)[0]
    assert (g[1] == 0).all() and g[2].isnan().all() and g[[0, 4]].isfinite().all()


def test_rows_apart_unaligned_and_folded():
    big, _ = make(64, 1100, "bf16", 2)
    big = big.cuda()
    for x in (big[:, :1000], big[:, 1:1000], big[::2, 3:700], big.t()[:900, :32], big[:1, :77].expand(6, 77)):
        t = torch.arange(x.shape[0], device="cuda") % x.shape[1]
        a, b = lm.token_logprobs(x, t, top=7), lm.token_logprobs(x.contiguous(), t, top=7)
        assert torch.equal(a.top_indices, b.top_indices) and torch.allclose(a.logprobs, b.logprobs, atol=1e-5) and torch.allclose(a.entropy, b.entropy, atol=1e-5)
        xd = x.detach().requires_grad_()
        g = torch.autograd.grad(lm.token_logprobs(xd, t).logprobs.sum(), xd)[0]
        yd = x.contiguous().detach().requires_grad_()
        k = torch.autograd.grad(lm.token_logprobs(yd, t).logprobs.sum(), yd)[0]
        assert torch.allclose(g.float(), k.float(), atol=2.0 ** -8)
    x = big[:60, :500].reshape(3, 20, 500)
    got = lm.token_logprobs(x, torch.zeros(3, 20, dtype=torch.int64, device="cuda"), top=4)
    assert got.logprobs.shape == got.entropy.shape == (3, 20) and got.top_indices.shape == got.top_logprobs.shape == (3, 20, 4)


def test_results_repeat_to_the_bit():
    x, t = make(3, 131072, "bf16", 3)
    x = (x * 4).round() / 4                         # many equal ones
    xd, td = x.cuda(), t.cuda()
    first = lm.token_logprobs(xd, td, top=32)
    for _ in range(10):
        again = lm.token_logprobs(xd, td, top=32)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    check(x, t, 32, first)


def test_rows_past_32_bits():
    rows, vocab = 70001, 65537                      # 4.6e9 logits
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    x[rows - 1, vocab - 1] = 30.0
    t = torch.full((rows,), vocab - 1, device="cuda")
    got = lm.token_logprobs(x, t, top=1)
    assert abs(float(got.logprobs[rows - 1])) < 1e-6 and int(got.top_indices[rows - 1]) == vocab - 1
    assert abs(float(got.logprobs[rows - 2]) + np.log(vocab)) < 1e-4 and int(got.top_indices[rows - 2]) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_raw_pointers(dtype):
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    rows, vocab, top = 9, 1001, 4
    x = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(1)).to(t).cuda().requires_grad_()
    targets = torch.arange(rows, device="cuda") * 100
    got = lm.token_logprobs(x, targets, top=top)
    dl, de = torch.linspace(-1, 1, rows, device="cuda"), torch.linspace(0.5, -0.5, rows, device="cuda")
    (dx,) = torch.autograd.grad((got.logprobs, got.entropy), x, (dl, de))
    lp, ent, stats, tops = (torch.empty(n, device="cuda") for n in (rows, rows, 2 * rows, rows * top))
    idx, out, st, p = torch.empty(rows * top, dtype=torch.int64, device="cuda"), torch.empty_like(dx), binding.current_stream_handle(), torch.Tensor.data_ptr
    binding.div_token_logprobs_forward(p(x), vocab, rows, vocab, dtype, p(targets), top, p(lp), p(ent), p(stats), p(tops), p(idx), st)
    binding.div_token_logprobs_backward(p(x), vocab, rows, vocab, dtype, p(targets), p(stats), p(ent), p(dl), p(de), p(out), st)
    assert torch.equal(lp, got.logprobs) and torch.equal(ent, got.entropy) and torch.equal(tops.view(rows, top), got.top_logprobs)
    assert torch.equal(idx.view(rows, top), got.top_indices) and torch.equal(out, dx)
