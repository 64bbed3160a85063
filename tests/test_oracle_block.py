"""Pins of the CPU oracle of the operators around the layer (oracle/block_oracle.py)."""
import numpy as np
import pytest

from oracle import block_oracle as bo

RNG = np.random.default_rng


def test_philox_known_answers():
    """The generator's published test vectors: all bits 0, all bits 1, digits of pi."""
    f = 0xFFFFFFFF
    for counter, key, want in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                               ((f, f, f, f), (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                               ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                                (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in bo.philox4x32_10(counter, key)) == want


def test_dropout_factor_rate_and_independence():
    T, H = 400, 1000
    for p in (0.1, 0.5):
        f = bo.dropout_factor(T, H, p, 1234567890123, 99)
        # a binomial's mean: five standard deviations
        assert abs((f == 0).mean() - p) < 5 * np.sqrt(p * (1 - p) / (T * H))
        for other in (bo.dropout_factor(T, H, p, 1234567890124, 99), bo.dropout_factor(T, H, p, 1234567890123, 100), np.roll(f, 1, 0),
                      np.roll(f, 1, 1)):
            both = ((f == 0) & (other == 0)).mean()
            assert abs(both - p * p) < 5 * np.sqrt(p * p * (1 - p * p) / (T * H))
    assert (bo.dropout_factor(3, 5, 0.0, 1, 2) == 1).all() and (bo.dropout_factor(3, 5, 1.0, 1, 2) == 0).all()


def differences(fn, x, h=1e-6):
    """Central differences of the scalar fn at x, element by element."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (fn(a) - fn(b)) / (2 * h)
    return g


@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_gradients_against_differences(affine):
    r = RNG(5)
    T, H = 4, 9
    x, dy = r.normal(size=(T, H)) + 0.7, r.normal(size=(T, H))
    gamma, beta = (r.normal(size=H), r.normal(size=H)) if affine else (None, None)
    _, mean, rstd = bo.layer_norm(x, gamma, beta, 1e-5)
    dx, dg, db = bo.layer_norm_backward(dy, x, gamma, mean, rstd)
    np.testing.assert_allclose(dx, differences(lambda a: (dy * bo.layer_norm(a, gamma, beta, 1e-5)[0]).sum(), x), atol=1e-7)
    if affine:
        np.testing.assert_allclose(dg, differences(lambda a: (dy * bo.layer_norm(x, a, beta, 1e-5)[0]).sum(), gamma), atol=1e-7)
        np.testing.assert_allclose(db, differences(lambda a: (dy * bo.layer_norm(x, gamma, a, 1e-5)[0]).sum(), beta), atol=1e-7)


@pytest.mark.parametrize("masked", [False, True])
def test_router_gradients_against_differences(masked):
    """Loss plus a linear function of the routing weights, both through the logits; the selection itself is held."""
    r = RNG(6)
    T, E, k, coef = 6, 7, 3, 0.37
    logits, dw = r.normal(size=(T, E)), r.normal(size=(T, k))
    idx = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    mask = np.array([1, 0, 1, 1, 0, 1]) if masked else None

    def weights(l):
        z = np.exp(np.take_along_axis(l, idx, 1))
        return z / z.sum(1, keepdims=True)

    counts, n, _, _ = bo.balance(logits, idx, mask, coef)
    d = bo.router_backward(logits, idx, weights(logits), dw, mask, coef, counts, n, dloss=2.5)
    want = differences(lambda l: 2.5 * bo.balance(l, idx, mask, coef)[3] + (dw * weights(l)).sum(), logits)
    np.testing.assert_allclose(d, want, atol=1e-8)


def test_balance_is_least_for_an_even_router():
    """Even counts and even probabilities give coef; one expert that takes all gives coef * E / k."""
    T, E, k = 12, 4, 2
    even = np.zeros((T, E))
    idx = np.array([[(t * k + j) % E for j in range(k)] for t in range(T)])
    assert np.isclose(bo.balance(even, idx, None, 0.5)[3], 0.5)
    sure = np.zeros((T, E))
    sure[:, 1] = 60.0
    assert np.isclose(bo.balance(sure, np.tile([1, 2], (T, 1)), None, 0.5)[3], 0.5 * E / k)
    assert bo.balance(even, idx, np.zeros(T), 0.5)[3] == 0.0
    assert (bo.router_probabilities(np.full((2, 3), -np.inf)) == 0).all()


def test_quantize_w4_takes_the_nearest_code():
    r = RNG(7)
    w = (r.normal(size=(2, 64, 5)) * np.exp(r.normal(size=(2, 64, 5)) * 2)).astype(np.float32)
    w[0, :32, 1] = 0.0
    q, s = bo.quantize_w4(w)
    back = bo.dequantize_w4(q, s)
    assert s[0, 0, 1] == 127 and (back[0, :32, 1] == 0).all()
    for e, g, n in np.ndindex(2, 2, 5):
        unit = 2.0 ** (int(s[e, g, n]) - 127)
        block = w[e, g * 32:(g + 1) * 32, n].astype(np.float64)
        if block.any():
            assert 4 * unit <= np.abs(block).max() < 8 * unit
        codes = np.concatenate([bo.E2M1, -bo.E2M1]) * unit
        best = np.abs(block[:, None] - codes).min(axis=1)
        np.testing.assert_allclose(np.abs(block - back[e, g * 32:(g + 1) * 32, n]), best, atol=1e-12 * unit)
    # halves: ties to the even code
    tie = np.zeros((1, 32, 1))
    tie[0, :9, 0] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0]
    got = bo.dequantize_w4(*bo.quantize_w4(tie))[0, :9, 0]
    np.testing.assert_array_equal(got, [4.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -4.0])
    bad = np.ones((1, 32, 2))
    bad[0, 3, 1] = np.inf
    q, s = bo.quantize_w4(bad)
    assert s[0, 0, 0] == 125 and s[0, 0, 1] == 255
