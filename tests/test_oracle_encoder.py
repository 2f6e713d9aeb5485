"""The float64 reference of the encoder's operators against closed forms, differences and torch."""
import numpy as np
import torch

from oracle import encoder_ref as R


def rng_of(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_norm_closed_forms():
    x = np.array([[[3.0, -4.0]], [[1.0, 1.0]]])
    y, t = R.rms_norm(x, np.array([1.0, 2.0]), eps=0.0)
    size = np.sqrt(12.5)
    assert np.allclose(y[0, 0], [3 / size, -8 / size], rtol=1e-15) and np.allclose(y[1, 0], [1, 2]) and np.array_equal(t, x)
    y, t = R.rms_norm(x, np.ones(2), -x, np.array([1, 0]))
    assert not y.any() and not t.any()
    y, _ = R.rms_norm(x, np.ones(2), None, np.array([2, 1]))
    assert np.isnan(y[0]).all() and np.isfinite(y[1]).all()


def test_norm_gradient_by_differences():
    rng = rng_of(1)
    x, r, w, dy, dsum = (rng.standard_normal(s) for s in ((2, 3, 5), (2, 3, 5), (5,), (2, 3, 5), (2, 3, 5)))
    lens = np.array([3, 1])

    def value(x, w):
        y, t = R.rms_norm(x, w, r, lens, 1e-2)
        return np.sum(y * dy) + np.sum(t * dsum)
    dx, dw, _, _ = R.rms_norm_grad(x + r, w, dy, dsum, lens, 1e-2)
    for got, at in ((dx, "x"), (dw, "w")):
        d = rng.standard_normal(got.shape)
        up, down = (value(x + e * d, w) if at == "x" else value(x, w + e * d) for e in (1e-5, -1e-5))
        assert abs(np.sum(got * d) - (up - down) / 2e-5) < 1e-7


def test_quantized_rows_and_their_product():
    x = np.array([[1.0, -2.0, 0.5], [0, 0, 0], [np.inf, 1, 1], [np.nan, 0, 0], [2.0 ** -101, 0, 0]])
    quotient, scale = R.quantize_rows(x)
    assert np.array_equal(quotient[0], [63.5, -127, 31.75]) and scale[0] == 2 / 127
    assert not quotient[1:].any() and scale[1] == 0 and np.isnan(scale[2:4]).all() and scale[4] == 0
    q, w = np.array([[1, -127, 3]]), np.array([[127, 127, 0], [0, 0, 5]])
    y, size = R.linear8(q, np.array([0.5]), w, np.array([2.0, 1.0]), np.array([1.0, -1.0]))
    assert np.array_equal(y, [[-126 * 127 + 1.0, 6.5]]) and np.array_equal(size, [[126 * 127 + 1.0, 8.5]])


def test_rotary_keeps_lengths_and_differences_of_positions():
    rng = rng_of(2)
    freq = 10000.0 ** (-np.arange(0, 6, 2) / 6)
    for inter in (False, True):
        a, b = rng.standard_normal((2, 1, 1, 1, 8))
        dots = []
        for p, q in ((0, 0), (5, 5), (100007, 100007)):
            u, v = R.rotary(a, freq, [p], None, inter)[0], R.rotary(b, freq, [q], None, inter)[0]
            assert np.isclose(np.linalg.norm(u), np.linalg.norm(a)) and np.array_equal(u[..., 6:], a[..., 6:])
            dots.append(np.sum(u * v))
        assert np.allclose(dots, dots[0])
        assert np.allclose(R.rotary(R.rotary(a, freq, [7], None, inter)[0], freq, [7], None, inter, -1.0)[0], a)
    x = np.zeros((1, 2, 1, 2))
    x[..., 0] = 1.0
    assert np.allclose(R.rotary(x, np.array([np.pi / 2]))[0][0, 1, 0], [0, 1])


def test_attention_against_torch_without_pages():
    rng = rng_of(3)
    B, L, Hq, Hkv, D, page = 2, 3, 4, 2, 5, 4
    q, k, v = (rng.standard_normal((B, L, h, D)) for h in (Hq, Hkv, Hkv))
    kc, vc = rng.standard_normal((2, 9, Hkv, page, D))
    pages, cached, lens = np.array([[3, 1, 8], [0, 7, 2]]), np.array([6, 2]), np.array([3, 2])
    for causal, left in ((True, None), (False, None), (True, 4), (False, 3), (True, 0)):
        out, _, _, ka, va = R.cached_attention(q, k, v, kc, vc, pages, cached, lens, causal=causal, left=left)
        for b in range(B):
            c, n = cached[b], lens[b]
            keys, values = (np.concatenate([a[pages[b]].transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :c + n]])
                            for a in (ka, va))
            at = c + np.arange(n)[:, None]
            j = np.arange(c + n)[None]
            seen = (j <= at if causal else j >= 0) & (True if left is None else j >= at - left)
            want = torch.nn.functional.scaled_dot_product_attention(
                torch.from_numpy(q[b, :n]).transpose(0, 1), torch.from_numpy(keys).repeat_interleave(2, 0),
                torch.from_numpy(values).repeat_interleave(2, 0), torch.from_numpy(np.broadcast_to(seen, (n, c + n)).copy()))
            assert np.allclose(out[b, :n], want.transpose(0, 1).numpy(), atol=1e-12) and not out[b, n:].any()
    assert np.isnan(R.cached_attention(q, k, v, kc, vc, pages, np.array([10, 0]), lens)[0][0]).all()
    bad = pages.copy()
    bad[0, 0] = 9
    out = R.cached_attention(q, k, v, kc, vc, bad, cached, lens, left=1)[0]
    assert np.isfinite(out).all()
    out = R.cached_attention(q, k, v, kc, vc, bad, cached, lens)[0]
    assert np.isnan(out[0]).all() and np.isfinite(out[1]).all()
