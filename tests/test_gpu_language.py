"""The operators of language models as they are used together: layers, a small model's training step, a captured decoding
step."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as lo
from paper_2208_04187_b200 import build
from paper_2208_04187_b200 import language as lm
from paper_2208_04187_b200.autograd import DivisionCache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built_library():
    build.build()


def f64(t):
    return t.detach().cpu().double().numpy()


def make(*shape, seed=0, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype)


def near(got, a, b, dtype):
    """A product of quantised operands: sums in 32 bits, one rounding."""
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    half = torch.finfo(dtype).eps / 2
    bound = a.shape[1] * 2.0 ** -23 * size
    assert (np.abs(f64(got) - want) <= bound + half * (np.abs(want) + bound)).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("m, k, n", [(1, 64, 96), (37, 100, 130), (256, 384, 128), (500, 65, 33)])
def test_linear_and_its_gradients(m, k, n, fmt):
    x, w, dy = make(m, k, seed=1), make(n, k, seed=2, dtype=torch.float32), make(m, n, seed=3)
    xd, wd = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    y = lm.mx_linear(xd, wd, fmt=fmt)
    q = lambda a: lo.mx_values(a, fmt)  # noqa: E731
    near(y, q(f64(x)), q(f64(w)), torch.bfloat16)
    dx, dw = torch.autograd.grad(y, (xd, wd), dy.cuda(), retain_graph=True)
    assert dx.dtype == torch.bfloat16 and dw.dtype == torch.float32
    near(dx, q(f64(dy)), q(f64(w).T), torch.bfloat16)
    near(dw, q(f64(dy).T), q(f64(x).T), torch.float32)
    # one of them alone
    assert torch.equal(torch.autograd.grad(lm.mx_linear(xd, w.cuda(), fmt=fmt), xd, dy.cuda())[0], dx)
    assert torch.equal(torch.autograd.grad(lm.mx_linear(x.cuda(), wd, fmt=fmt), wd, dy.cuda())[0], dw)
    three = lm.mx_linear(xd.view(m, 1, k), wd, fmt=fmt)
    assert torch.equal(three.view(m, n), y)


def test_what_a_linear_layer_keeps():
    x = make(4096, 2048, seed=1).cuda().requires_grad_()
    w = make(2048, 2048, seed=2).cuda().requires_grad_()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = lm.mx_linear(x, w, fmt="e2m1")
    kept = torch.cuda.memory_allocated() - before - y.numel() * 2
    assert kept <= (x.numel() + w.numel()) * 4.25 / 8 * 1.02


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
@pytest.mark.parametrize("fused", [False, True])
def test_norm_and_linear_in_one(fmt, fused):
    x, r, g, w = make(70, 200, seed=1).cuda(), make(70, 200, seed=2).cuda(), (1 + make(200, seed=3, scale=0.1)).cuda(), make(150, 200, seed=4).cuda()
    args = [t.requires_grad_() for t in (x, g, w)] + ([r.requires_grad_()] if fused else [])
    out, h = lm.mx_norm_linear(x, g, w, r if fused else None, eps=1e-5, fmt=fmt)
    q, h2 = lm.rms_norm_mx(x, g, r if fused else None, eps=1e-5, fmt=fmt)
    assert torch.equal(h, h2) and torch.equal(out, lm.mx_matmul(q, lm.mx_quantize(w, fmt)))
    do, dh = make(70, 150, seed=5).cuda(), make(70, 200, seed=6).cuda()
    got = torch.autograd.grad((out, h) if fused else out, args, (do, dh) if fused else do)
    # the same from its parts
    y, h3 = lm.rms_norm(x, g, r if fused else None, eps=1e-5)
    dy = lm.mx_matmul(lm.mx_quantize(do, fmt), lm.mx_quantize_columns(w, fmt))
    parts = torch.autograd.grad((y, h3) if fused else y, [args[0], args[1]] + args[3:], (dy, dh) if fused else dy)
    assert torch.equal(got[0], parts[0]) and torch.equal(got[1], parts[1])
    assert torch.equal(got[2], lm.mx_matmul(lm.mx_quantize_columns(do, fmt), lm.mx_quantize_columns(y, fmt)))
    if fused:
        assert torch.equal(got[3], parts[2])


class Block(torch.nn.Module):
    def __init__(self, d, fmt):
        super().__init__()
        self.up = lm.DivisionNormLinear(d, 2 * d, fmt=fmt, device="cuda", dtype=torch.bfloat16)
        self.down = lm.DivisionLinear(2 * d, d, fmt=fmt, device="cuda", dtype=torch.bfloat16)

    def forward(self, x, h):
        out, h = self.up(x, h)
        return self.down(torch.relu(out)), h


class Model(torch.nn.Module):
    def __init__(self, vocab, d, layers, fmt):
        super().__init__()
        self.embed = torch.nn.Embedding(vocab, d, device="cuda", dtype=torch.bfloat16)
        self.blocks = torch.nn.ModuleList(Block(d, fmt) for _ in range(layers))
        self.norm = lm.DivisionRMSNorm(d, device="cuda", dtype=torch.bfloat16)
        self.head = lm.DivisionLinear(d, vocab, bias=False, fmt=fmt, device="cuda", dtype=torch.bfloat16)

    def forward(self, tokens):
        h = self.embed(tokens)
        x = torch.zeros_like(h)
        for b in self.blocks:
            x, h = b(x, h)
        y, _ = self.norm(x, h)
        return self.head(y)


@pytest.mark.parametrize("fmt", ["e4m3", "e2m1"])
def test_a_training_step(fmt):
    torch.manual_seed(0)
    model = Model(501, 96, 2, fmt)
    tokens = torch.randint(0, 501, (4, 33), device="cuda")
    got = lm.token_logprobs(model(tokens[:, :-1]), tokens[:, 1:])
    loss = -got.logprobs.mean() - 0.01 * got.entropy.mean()
    loss.backward()
    grads = [p.grad for p in model.parameters()]
    assert all(g is not None and g.shape == p.shape and g.isfinite().all() and g.abs().sum() > 0 for g, p in zip(grads, model.parameters()))
    # and again, to the bit (embeddings are summed by torch in no fixed order)
    model.zero_grad()
    got = lm.token_logprobs(model(tokens[:, :-1]), tokens[:, 1:])
    (-got.logprobs.mean() - 0.01 * got.entropy.mean()).backward()
    assert all(torch.equal(a, p.grad) for a, (name, p) in zip(grads, model.named_parameters()) if "embed" not in name)


def test_the_gradient_of_a_model_is_near_that_of_the_same_model_in_full_precision():
    """Quantisation errors are at most half a step: 2^-4 of a number's block's largest with e4m3 (2^-4 of the number itself where it is
    normal).  The product of two such operands is off by less than 2 * 2^-4 + 2^-8 of the sum of magnitudes."""
    x, w = make(64, 256, seed=1), make(80, 256, seed=2)
    y = lm.mx_linear(x.cuda(), w.cuda())
    want, size = f64(x) @ f64(w).T, np.abs(f64(x)) @ np.abs(f64(w)).T
    assert (np.abs(f64(y) - want) <= (2 * 2.0 ** -4 + 2.0 ** -8) * size * (1 + 2.0 ** -8) + 2.0 ** -9 * np.abs(want) + 0.05).all()


def test_a_decoding_step_is_captured_and_replayed():
    """Norm -> 4-bit product -> log probabilities, for one token, on buffers whose contents change."""
    d, vocab = 512, 3000
    g = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    w = lm.mx_quantize(make(vocab, d, seed=1).cuda(), "e2m1")
    x, h = make(1, d, seed=2).cuda(), make(1, d, seed=3).cuda()
    target = torch.tensor([17], device="cuda")

    def step():
        q, k = lm.rms_norm_mx(x, g, h, fmt="e2m1")
        return (k, *lm.token_logprobs(lm.mx_matmul(q, w), target, top=8))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        x.copy_(make(1, d, seed=10 + seed).cuda())
        h.copy_(make(1, d, seed=20 + seed).cuda())
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_two_streams_at_once():
    xs = [make(300, 1024, seed=i).cuda() for i in range(4)]
    w = lm.mx_quantize(make(700, 1024, seed=9).cuda(), "e4m3")
    g = torch.ones(1024, device="cuda", dtype=torch.bfloat16)
    t = torch.arange(300, device="cuda")

    def chain(x):
        q, _ = lm.rms_norm_mx(x, g)
        return lm.token_logprobs(lm.mx_matmul(q, w), t, top=3)
    want = [chain(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(5):
        got = []
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(chain(x))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(got, want) for a, b in zip(p, q))


def test_a_gradient_has_no_gradient():
    x, w = make(8, 64, seed=1).cuda().requires_grad_(), make(16, 64, seed=2).cuda().requires_grad_()
    t = torch.arange(8, device="cuda")
    for y in (lm.mx_linear(x, w), lm.rms_norm(x, w[0])[0], lm.token_logprobs(x, t).logprobs, lm.mx_norm_linear(x, w[0], w)[0]):
        (g,) = torch.autograd.grad(y.float().sum(), x, create_graph=True)
        assert g.isfinite().all()
        with pytest.raises(RuntimeError, match="has no gradient"):
            g.float().sum().backward()


def test_a_training_step_is_captured_and_replayed():
    """Forward and backward in one graph (no eager graph of the same leaves is alive: torch would tie the legacy stream to the capture)."""
    d, vocab = 128, 300
    g, w = torch.ones(d, device="cuda", dtype=torch.bfloat16).requires_grad_(), make(vocab, d, seed=1).cuda().requires_grad_()
    x, t = make(40, d, seed=2).cuda().requires_grad_(), torch.arange(40, device="cuda")
    dl = torch.full((40,), -1 / 40, device="cuda")

    def step():
        out, _ = lm.mx_norm_linear(x, g, w)
        got = lm.token_logprobs(out, t)
        return (got.logprobs, *torch.autograd.grad(got.logprobs, (x, g, w), dl))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    with torch.no_grad():
        x.copy_(make(40, d, seed=3).cuda())
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_saved_tensors_are_watched():
    x, g = make(8, 64, seed=1).cuda().requires_grad_(), torch.ones(64, device="cuda", dtype=torch.bfloat16)
    z = x * 1
    y, _ = lm.rms_norm(z, g)
    z.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()
    z = x * 1
    w = make(16, 64, seed=2).cuda()
    y = lm.mx_linear(z, w.requires_grad_())
    with torch.no_grad():
        z.zero_()                                       # (its quantised form alone is kept)
    dw = torch.autograd.grad(y.float().sum(), w)[0]
    assert dw.abs().sum() > 0


def test_forward_mode_derivatives_are_refused():
    """A tensor with a tangent need not ask for a gradient: an output without a tangent would say that the derivative is 0."""
    forward_ad = torch.autograd.forward_ad
    x, g, w = make(8, 64, seed=1).cuda(), make(64, seed=2).cuda(), make(16, 64, seed=3).cuda()
    t = torch.arange(8, device="cuda")
    calls = [lambda x, r, g, w: lm.mx_linear(x, w), lambda x, r, g, w: lm.rms_norm(x, g, r)[0], lambda x, r, g, w: lm.mx_norm_linear(x, g, w, r)[0]]
    takes = [(0, 3), (0, 1, 2), (0, 1, 2, 3)]
    with forward_ad.dual_level():
        for call, which in zip(calls, takes):
            for i in which:
                args = [x, x, g, w]
                args[i] = forward_ad.make_dual(args[i], torch.ones_like(args[i]))
                for grad in (True, False):
                    with torch.set_grad_enabled(grad), pytest.raises(NotImplementedError, match="forward-mode"):
                        call(*args)
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            lm.token_logprobs(dual, t)
        with torch.inference_mode():                                   # (where torch passes no tangents on either)
            assert torch.equal(lm.token_logprobs(dual, t).logprobs, lm.token_logprobs(x, t).logprobs)
        for call in calls:                                             # no tangent, no refusal
            call(x, x, g, w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_a_replaced_norm_gives_what_torchs_gave(dtype):
    """Without an epsilon of its own, on rows so small that it decides."""
    norm = torch.nn.RMSNorm(64, device="cuda", dtype=dtype)
    x = make(5, 64, seed=1, scale=0.01, dtype=dtype).cuda()
    want = norm(x)
    got = lm.to_division_layers(torch.nn.Sequential(norm))[0](x)
    # both: a sum of 64 and a handful of operations in 32 bits, then half a step
    size = want.double().abs()
    assert ((got.double() - want.double()).abs() <= 2 * (torch.finfo(dtype).eps / 2 + 40 * 2.0 ** -24) * (1 + 2.0 ** -8) * size).all()


@pytest.mark.parametrize("fused", [False, True])
def test_a_norm_under_the_activation_cache(fused):
    """What a norm keeps of a map of 3 dimensions is a map of 3 dimensions: the cache takes it, and the gradients are the formula's at the map that
    comes back."""
    b, t, d = 4, 64, 256
    x, w = make(b, t, d, seed=1, dtype=torch.float32).cuda().requires_grad_(), (1 + make(d, seed=2, scale=0.1, dtype=torch.float32)).cuda().requires_grad_()
    r = make(b, t, d, seed=3, dtype=torch.float32).cuda().requires_grad_() if fused else None
    dy = make(b, t, d, seed=4, dtype=torch.float32).cuda()
    back = []

    class Watched(DivisionCache):
        def unpack(self, h):
            back.append(super().unpack(h))
            return back[-1]
    with Watched(block=8, qbits=8) as cache:
        y, h = lm.rms_norm(x * 1, w, r, eps=1e-5)
    assert cache.maps == 1 and y.shape == h.shape == (b, t, d)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    (kept,) = [u for u in back if u.shape == (b, t, d)]
    assert not torch.equal(kept, h) and kept.isfinite().all()
    n64 = f64(h).reshape(-1, d)
    rstd = 1 / np.sqrt((n64 * n64).mean(1) + 1e-5)
    want, want_w = lo.rms_norm_backward(f64(dy).reshape(-1, d), None, f64(kept).reshape(-1, d), f64(w), rstd)
    # every term of a sum to 300 steps in 32 bits (no sum here has more)
    size = rstd[:, None] * np.abs(f64(dy).reshape(-1, d) * f64(w))
    n = np.abs(f64(kept).reshape(-1, d)) * rstd[:, None]
    bound = size + n * (size * n).mean(1, keepdims=True)
    assert (np.abs(f64(dx).reshape(-1, d) - want) <= 300 * 2.0 ** -24 * bound).all()
    assert (np.abs(f64(dw) - want_w) <= 300 * 2.0 ** -24 * (np.abs(f64(dy).reshape(-1, d)) * n).sum(0)).all()


def test_shapes_of_norms_and_layers():
    """Outputs and gradients have the shapes of what was given, rows apart or folded."""
    d = 96
    g, w = torch.ones(d, device="cuda", dtype=torch.bfloat16).requires_grad_(), make(40, d, seed=1).cuda().requires_grad_()
    for shape in ((d,), (5, d), (2, 3, d), (2, 1, 3, d)):
        x, r = make(*shape, seed=2).cuda().requires_grad_(), make(*shape, seed=3).cuda().requires_grad_()
        for residual in (None, r):
            y, h = lm.rms_norm(x, g, residual)
            out, k = lm.mx_norm_linear(x, g, w, residual)
            q, z = lm.rms_norm_mx(x, g, residual)
            assert y.shape == h.shape == k.shape == z.shape == shape and out.shape == shape[:-1] + (40,) and torch.equal(h, k) and torch.equal(h, z)
            assert q.shape == (x.numel() // d, d) and torch.equal(lm.mx_matmul(q, lm.mx_quantize(w)), out.view(-1, 40))
            flat, _ = lm.rms_norm(x.detach().reshape(-1, d), g, None if residual is None else residual.detach().reshape(-1, d))
            assert torch.equal(y.view(-1, d), flat)
            leaves = [x, g] + ([r] if residual is not None else [])
            for o in (y, out):
                for leaf, grad in zip(leaves, torch.autograd.grad((o.float() * torch.arange(o.size(-1), device="cuda")).sum(), leaves)):
                    assert grad.shape == leaf.shape and grad.isfinite().all() and grad.abs().sum() > 0
            h.mul_(1) if residual is not None else None              # (no view that torch would forbid to change)
    a, b = make(6, 5, d, seed=4).cuda().transpose(0, 1), make(6, 5, 2 * d, seed=5).cuda()[..., :d].transpose(0, 1)
    y, h = lm.rms_norm(a, g, b)
    z, k = lm.rms_norm(a.contiguous(), g, b.contiguous())
    assert torch.equal(y, z) and torch.equal(h, k)


@pytest.mark.parametrize("fused", [False, True])
def test_a_frozen_norm_costs_its_layer_nothing(fused):
    """Where the weight alone wants a gradient, neither the weight's columns are kept nor a gradient of the norm made."""
    m, d, n = 512, 1024, 2048
    x, g, w = make(m, d, seed=1).cuda(), (1 + make(d, seed=2, scale=0.1)).cuda(), make(n, d, seed=3).cuda()
    r, dy = make(m, d, seed=4).cuda() if fused else None, make(m, n, seed=5).cuda()

    def kept(*leaves):
        for t in leaves:
            t.requires_grad_()
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        out, h = lm.mx_norm_linear(x, g, w, r, fmt="e4m3")
        size = torch.cuda.memory_allocated() - before - 2 * out.numel() - (2 * h.numel() if fused else 0)
        grads = torch.autograd.grad(out, leaves, dy)
        for t in leaves:
            t.requires_grad_(False)
        return size, grads
    alone, (dw,) = kept(w)
    both, (dw2, dg) = kept(w, g)
    assert torch.equal(dw, dw2) and dg.abs().sum() > 0
    blob = n * d * 33 // 32
    assert alone <= 16 * 1024 and both >= blob                    # alone: a number a row
    # a leaf that this call does not ask for
    w.requires_grad_(), x.requires_grad_()
    out, _ = lm.mx_norm_linear(x, g, w, r, fmt="e4m3")
    assert torch.equal(torch.autograd.grad(out, w, dy, retain_graph=True)[0], dw)
    dx = torch.autograd.grad(out, x, dy)[0]
    assert dx.shape == x.shape and dx.abs().sum() > 0
