"""Pins of the oracle for the operators of a training step: published vectors of the generator, finite differences of the
losses it differentiates, invariants of the formulas."""
import numpy as np
import pytest

from oracle import training_operators as op


def test_philox_published_vectors():
    # the known answers that the generator's authors give for ten rounds
    assert op.philox4x32_10((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert op.philox4x32_10((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert op.philox4x32_10((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_share_and_extremes():
    kept, scale = op.dropout_kept(64, 128, 7, 9, 0.25)
    assert scale == 4.0 / 3.0
    assert abs(kept.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / kept.size)
    assert op.dropout_kept(2, 20, 1, 2, 0.0)[0].all() and not op.dropout_kept(2, 20, 1, 2, 1.0)[0].any()
    assert not np.array_equal(kept, op.dropout_kept(64, 128, 7, 10, 0.25)[0])
    assert np.array_equal(kept[3:, :77], op.dropout_kept(61, 77, 7, 9, 0.25, first_row=3)[0])     # a value's bits go by its row and column


def differences(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = h
        g[i] = (f(x + d) - f(x - d)) / (2 * h)
    return g


@pytest.mark.parametrize("rotated,halves", [(0, False), (6, False), (8, True), (4, True)])
def test_norm_gradients_are_those_of_differences(rotated, halves):
    g = np.random.default_rng(3)
    x, dy, gain = g.standard_normal((2, 3, 2, 8)), g.standard_normal((2, 3, 2, 8)), 1 + 0.3 * g.standard_normal(8)
    pos = np.array([[0, 5, 9], [2, 100, 7]])
    kw = dict(positions=pos, eps=1e-2, base=100.0, rotated=rotated, halves=halves, scale=0.7)
    dx, dg = op.qk_norm_backward(x, dy, gain, **kw)
    assert np.abs(dx - differences(lambda v: (op.qk_norm(v, gain, **kw) * dy).sum(), x)).max() < 1e-7
    assert np.abs(dg - differences(lambda v: (op.qk_norm(x, v, **kw) * dy).sum(), gain)).max() < 1e-7


def test_rotation_keeps_lengths_and_depends_on_distances():
    g = np.random.default_rng(5)
    a, b = g.standard_normal((1, 2, 1, 16)), g.standard_normal((1, 2, 1, 16))
    for halves in (False, True):
        turn = lambda v, p: op.rotate(v, np.array([p]), 10000.0, 16, halves)
        assert np.allclose((turn(a, [3, 8]) ** 2).sum(-1), (a ** 2).sum(-1))
        dots = [(turn(a, [p, p]) * turn(b, [p + 5, p + 9])).sum(-1) for p in (0, 11)]
        assert np.allclose(*dots)
        assert np.allclose(op.rotate(turn(a, [3, 8]), np.array([[3, 8]]), 10000.0, 16, halves, back=True), a)


@pytest.mark.parametrize("kind", ["counts", "entropy"])
def test_balance_gradient_is_that_of_differences(kind):
    g = np.random.default_rng(11)
    z = g.standard_normal((6, 2, 2, 5))
    idx = np.argsort(-z, axis=-1)[..., :2].transpose(1, 0, 2, 3)
    mask = np.array([1, 1, 0, 1, 1, 0])
    loss, counts, P, dz = op.balance(z, idx, kind, 0.3, mask)
    assert np.abs(dz - differences(lambda v: op.balance(v, idx, kind, 0.3, mask)[0], z)).max() < 1e-8
    assert (counts.sum(-1) == 8).all() and np.allclose(P.sum(-1), 1.0)
    assert not dz[2].any() and np.abs(dz.sum(-1)).max() < 1e-12


def test_balance_extremes():
    even = np.zeros((8, 1, 1, 4))
    idx = (np.arange(8)[None, :, None, None] + np.arange(2)) % 4
    assert np.isclose(op.balance(even, idx, "counts", 1.0)[0], 1.0)
    assert np.isclose(op.balance(even, idx, "entropy", 1.0)[0], -np.log(4))
    none = op.balance(even, idx, "counts", 1.0, np.zeros(8))
    assert none[0] == 0 and not none[1].any() and not none[2].any() and not none[3].any()
