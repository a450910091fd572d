"""The 64-bit statement of the language operators against properties that do not depend on it: tables of the number
formats, finite differences, and torch's own functions on the CPU."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as lo


def test_formats_hold_their_own_numbers():
    e2m1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    row = np.concatenate([e2m1, -e2m1, e2m1, -e2m1])[None]
    for power in (-100, -3, 0, 5, 90):
        assert np.array_equal(lo.mx_values(row * 2.0 ** power, "e2m1"), row * 2.0 ** power)
    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    e4m3 = e4m3[np.isfinite(e4m3)]
    pad = np.full((1, 8 * 32), 448.0)                       # every block's largest is the format's
    for b in range(8):
        part = e4m3[b * 32:b * 32 + 31]
        pad[0, b * 32:b * 32 + len(part)] = part
    assert np.array_equal(lo.mx_values(pad, "e4m3"), pad)


@pytest.mark.parametrize("fmt, borders", [("e2m1", {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0, 0.2501: 0.5, 4.99: 4.0, 5.01: 6.0}),
                                          ("e4m3", {232.0: 224.0, 1.0625: 1.0, 1.1875: 1.25, 2.0 ** -10: 0.0, 1.5 * 2.0 ** -9: 2.0 ** -8})])
def test_ties_go_to_even(fmt, borders):
    for value, want in borders.items():
        row = np.zeros((1, 32))
        row[0, 0], row[0, 1] = lo.LARGEST[fmt], value
        assert lo.mx_values(row, fmt)[0, 1] == want, value


def test_scales_are_the_smallest_that_clip_nothing():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp(4 * rng.standard_normal((50, 1)))
    for fmt in lo.LARGEST:
        _, s = lo.mx_blocks(x, fmt)
        big = np.abs(x.reshape(50, 2, 32)).max(2)
        assert (big <= s * lo.LARGEST[fmt]).all() and (big > s / 2 * lo.LARGEST[fmt]).all()


def test_rounding_agrees_with_torch():
    x = np.random.default_rng(1).standard_normal(1000) * 10.0 ** np.random.default_rng(2).integers(-39, 38, 1000)
    x = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(lo.round_to(x, "bf16"), torch.from_numpy(x).float().bfloat16().double().numpy())
    small = x[np.abs(x) < 60000]
    assert np.array_equal(lo.round_to(small, "f16"), torch.from_numpy(small).half().double().numpy())


def _difference(f, x, i, j, d=1e-6):
    a, b = x.copy(), x.copy()
    a[i, j] += d
    b[i, j] -= d
    return (f(a) - f(b)) / (2 * d)


def test_norm_gradients_are_differences():
    rng = np.random.default_rng(3)
    x, w, dy, dh = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))

    def loss(x, w=w):
        y, h, _ = lo.rms_norm(x, None, w, 1e-5, "f64")
        return (y * dy).sum() + (h * dh).sum()
    _, h, rstd = lo.rms_norm(x, None, w, 1e-5, "f64")
    dx, dw = lo.rms_norm_backward(dy, dh, h, w, rstd)
    for i in range(3):
        for j in range(7):
            assert abs(_difference(loss, x, i, j) - dx[i, j]) < 1e-7
    for j in range(7):
        assert abs(_difference(lambda v: loss(x, v[0]), w[None], 0, j) - dw[j]) < 1e-7


def test_logprobs_agree_with_torch_and_differences():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((4, 11)) * 3
    x[1, 3:6] = -np.inf
    t = np.array([2, 7, -1, 10])
    lp, ent, top, idx = lo.token_logprobs(x, t, 4)
    ref = torch.log_softmax(torch.from_numpy(x), 1)
    p = ref.exp()
    assert np.allclose(lp[[0, 1, 3]], ref.numpy()[[0, 1, 3], [2, 7, 10]], atol=1e-14) and lp[2] == 0
    assert np.allclose(ent, -torch.xlogy(p, p).sum(1).numpy(), atol=1e-14)
    want, order = torch.topk(ref, 4, dim=1)
    assert np.allclose(top, want.numpy()) and np.array_equal(idx, order.numpy())
    dl, de = rng.standard_normal(4), rng.standard_normal(4)
    g = lo.token_logprobs_backward(x, t, dl, de)

    def loss(x):
        a, b, _, _ = lo.token_logprobs(x, t, 0)
        return (a * dl).sum() + (b * de).sum()
    for i in range(4):
        for j in range(11):
            if np.isfinite(x[i, j]):
                assert abs(_difference(loss, x, i, j) - g[i, j]) < 1e-7
            else:
                assert g[i, j] == 0


def test_equal_logits_go_by_index_and_empty_rows_have_nothing():
    x = np.array([[1.0, 5, 5, 1, 5], [-np.inf] * 5, [np.nan, 1, 2, np.nan, 0]])
    lp, ent, top, idx = lo.token_logprobs(x, [1, 0, 1], 3)
    assert idx[0].tolist() == [1, 2, 4] and idx[1].tolist() == [0, 1, 2] and idx[2].tolist() == [0, 3, 2]
    assert lp[1] == -np.inf and ent[1] == 0 and (top[1] == -np.inf).all()
    assert np.isnan(lp[2]) and np.isnan(ent[2]) and np.isnan(top[2]).all()
    assert (lo.token_logprobs_backward(x[:2], [1, 0], [1.0, 1.0], [1.0, 1.0])[1] == 0).all()
