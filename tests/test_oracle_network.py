"""The float64 reference of the network operators, pinned by closed forms, by differences and
by the published vectors of the generator."""
import numpy as np
import pytest

from oracle import network_ref as R


def test_philox_known_answers():
    # the all-zero and the digits-of-pi vectors of the generator's authors
    assert R.philox4x32([0] * 4, [0] * 2, 7) == [0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48]
    assert R.philox4x32([0] * 4, [0] * 2, 10) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert R.philox4x32([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0], 10) == [
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_dropout_numbers():
    # every 16-bit half of a block in turn, and a mask that may start anywhere
    words = R.philox4x32([5, 0, 3, 0], [7, 0], 7)
    got = [R.random16(40 + i, 7, 3) for i in range(8)]
    assert got == [w >> s & 0xffff for w in words for s in (0, 16)]
    full = R.keep_mask((64,), 0.4, -9, 1 << 40)
    assert np.array_equal(full[13:30], R.keep_mask((17,), 0.4, -9, 1 << 40, 13))
    assert R.threshold(0.0) == 0 and R.threshold(0.5) == 32768 and R.threshold(0.9999999) == 65535
    # 20000 draws at p = 0.3: six standard deviations of the mean are 0.0195
    assert abs(1.0 - R.keep_mask((20000,), 0.3, 1, 2).mean() - 0.3) < 0.02
    y = R.dropout(np.array([np.nan] * 64), 0.5, 3, 4)
    assert (y == 0).any() and np.isnan(y).any()


def test_recurrence_closed_forms():
    x = np.full((1, 6, 1), 2.0)
    h, last = R.gated_recurrence(x, np.zeros((1, 6, 1)), np.full((1, 1), 4.0))
    assert np.allclose(h[0, :, 0], 2.0 + 2.0 * 0.5 ** np.arange(1, 7)) and last[0, 0] == h[0, -1, 0]
    h, last = R.gated_recurrence(x, np.full((1, 6, 1), 1000.0), np.full((1, 1), 4.0))
    assert np.all(h == 4.0)
    h, last = R.gated_recurrence(x, np.full((1, 6, 1), -1000.0), np.full((1, 1), 4.0), np.array([3]))
    assert np.all(h[0, :3] == 2.0) and np.all(h[0, 3:] == 0.0) and last[0, 0] == 2.0
    h, last = R.gated_recurrence(x, x, np.full((1, 1), 4.0), np.array([0]))
    assert np.all(h == 0.0) and last[0, 0] == 4.0
    h, last = R.gated_recurrence(x, x, None, np.array([7]))
    assert np.isnan(h).all() and np.isnan(last).all()


def differences(f, args, grads, names, eps=1e-6):
    """Directional differences of the scalar f along random directions against the gradients."""
    rng = np.random.Generator(np.random.PCG64(5))
    for i, (a, g, name) in enumerate(zip(args, grads, names)):
        d = rng.standard_normal(a.shape)
        up, down = list(args), list(args)
        up[i], down[i] = a + eps * d, a - eps * d
        want = (f(*up) - f(*down)) / (2 * eps)
        assert abs(np.sum(g * d) - want) <= 1e-7 * (1.0 + abs(want)), name


def test_recurrence_gradient_differences():
    rng = np.random.Generator(np.random.PCG64(1))
    x, z, h0 = rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 3))
    dh, dl, lens = rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 3)), np.array([9, 4])

    def f(x, z, h0):
        h, last = R.gated_recurrence(x, z, h0, lens)
        return np.sum(h * dh) + np.sum(last * dl)
    differences(f, (x, z, h0), R.gated_recurrence_grad(x, z, dh, dl, h0, lens), ("x", "z", "h0"))
    for b, n in enumerate(lens):
        assert np.all(R.gated_recurrence_grad(x, z, dh, dl, h0, lens)[0][b, n:] == 0)


@pytest.mark.parametrize("act", ["relu", "tanh"])
def test_joint_gradient_differences(act):
    rng = np.random.Generator(np.random.PCG64(2))
    enc, pred = rng.standard_normal((2, 4, 5)), rng.standard_normal((2, 3, 5))
    tl, ul = np.array([4, 2]), np.array([1, 2])
    dh = rng.standard_normal((2, 4, 3, 5))

    def f(enc, pred):
        return np.sum(R.joint_hidden(enc, pred, tl, ul, act, 0.3, 11, 12) * dh)
    h, denc, dpred, _, _ = R.joint_hidden(enc, pred, tl, ul, act, 0.3, 11, 12, dh)
    differences(f, (enc, pred), (denc, dpred), ("enc", "pred"))
    assert np.all(h[0, :, 2:] == 0) and np.all(h[1, 2:] == 0)
    # the joint's dropout is the dropout of the whole tensor
    plain = R.joint_hidden(enc, pred, tl, ul, act)
    assert np.allclose(h, R.dropout(plain, 0.3, 11, 12), rtol=1e-15)


def test_embedding_gradient_differences():
    rng = np.random.Generator(np.random.PCG64(3))
    W, labels = rng.standard_normal((6, 4)), rng.integers(0, 6, size=(3, 5))
    lens, dout = np.array([5, 0, 2]), rng.standard_normal((3, 6, 4))

    def f(W):
        return np.sum(R.label_embedding(labels, W, lens, 1.5, 0) * dout)
    differences(f, (W,), (R.label_embedding_grad(labels, 6, dout, lens, 1.5, 0)[0],), ("weight",))
    out = R.label_embedding(np.array([[1, -1, 6]]), W)
    assert np.array_equal(out[0, 0], W[1]) and np.isnan(out[0, 1:]).all()
    assert np.isnan(R.label_embedding(labels, W, np.array([6, -1, 2]))[:2]).all()
