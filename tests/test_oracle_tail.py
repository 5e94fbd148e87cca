"""Pins of the oracle's model tail: closed forms and hand-written cases."""
import numpy as np
import pytest

from oracle import tail


def test_rms_norm_closed_forms():
    # equal entries normalise to their sign, whatever their size
    h, n = tail.residual_norm(None, np.full((1, 7), -3.0), None, None, None, 1e-30, 1.0)
    assert np.allclose(n, -1) and np.array_equal(h, np.full((1, 7), -3.0))
    # (3, 4): mean square 12.5
    _, n = tail.residual_norm(None, np.array([[3.0, 4.0]]), None, None, np.array([2.0, 1.0]),
                              0.0, 1.0)
    assert np.allclose(n, [[6 / np.sqrt(12.5), 4 / np.sqrt(12.5)]])
    # eps alone under a zero row
    _, n = tail.residual_norm(None, np.zeros((1, 3)), None, None, None, 4.0, 1.0)
    assert np.array_equal(n, np.zeros((1, 3)))


def test_residual_step_terms():
    y, h = np.array([[1.0, 1.0]]), np.array([[10.0, 20.0]])
    g, wp = np.array([[0.5, 2.0]]), np.array([3.0, 5.0])
    h1, _ = tail.residual_norm(y, h, g, wp, None, 0.0, 0.1)     # rms(y) = (1, 1)
    assert np.allclose(h1, [[10 + 0.1 * 0.5 * 3, 20 + 0.1 * 2 * 5]])
    h1, n = tail.residual_norm(y, h, None, None, None, 0.0, -1.0)
    assert np.allclose(h1, [[9, 19]])
    assert np.allclose((n ** 2).mean(), 1)


def test_e2m1_values_and_layout():
    assert [tail.e2m1(c) for c in range(8)] == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert all(tail.e2m1(c + 8) == -tail.e2m1(c) for c in range(8))
    codes = np.zeros((1, 32), dtype=np.uint8)
    codes[0, 0] = 0x21                   # element 0: code 1, element 1: code 2
    codes[0, 16] = 0x0f                  # element 32 (second group): code 15
    w = tail.mx4_weights(codes, np.array([[128, 125]], dtype=np.uint8))
    assert w[0, 0] == 1.0 and w[0, 1] == 2.0 and w[0, 32] == -1.5
    assert np.count_nonzero(w) == 3
    assert np.isnan(tail.mx4_weights(codes, np.array([[255, 127]], dtype=np.uint8))[0, :32]).all()


def test_history_by_hand():
    seen, count = tail.history([4, 4, 7, 4, 7, 9, -1, 50], 2, 5, 10)
    assert sorted(np.flatnonzero(seen)) == [4, 7]
    assert count[4] == 1 and count[7] == 2 and count.sum() == 3


def test_rules_by_hand():
    z = np.array([2.0, -2.0, 2.0, 2.0, np.nan, -np.inf])
    seen = np.array([1, 1, 0, 0, 0, 1], dtype=bool)
    count = np.array([3, 0, 0, 0, 0, 1])
    bias = np.array([0, 0, 0, -np.inf, 0, 0])
    allowed = np.array([1, 1, 1, 1, 0, 1], dtype=bool)
    out = tail.rule_logits(z, seen, count, bias, bias != 0, (2.0, 0.25, 0.5), allowed)
    assert list(out) == [1 - 0.25 - 1.5, -4.0, 2.0, -np.inf, -np.inf, -np.inf]
    xhat, p = tail.predict(np.stack([out, np.full(6, -np.inf)]))
    assert list(xhat) == [2, -1] and p[1] == 0
    assert p[0] == pytest.approx(1 / (1 + np.exp(-2.75) + np.exp(-6.0)))
