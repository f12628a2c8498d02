"""Pins of oracle/muon_oracle.py: the iteration's closed form on the singular values, from either side, and limits."""
import numpy as np
import pytest

from oracle.muon_oracle import A, B, C, muon_step, newton_schulz


def _by_svd(g, steps, eps=1e-7):
    u, s, v = np.linalg.svd(g, full_matrices=False)
    s = s / (np.linalg.norm(g) + eps)
    for _ in range(steps):
        s = A * s + B * s**3 + C * s**5
    return (u * s) @ v


@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (7, 1), (12, 12), (9, 30), (30, 9)])
@pytest.mark.parametrize("steps", [1, 5])
def test_closed_form_on_the_singular_values(shape, steps):
    g = np.random.default_rng(sum(shape)).normal(0, 3e-4, shape)
    np.testing.assert_allclose(newton_schulz(g, steps), _by_svd(g, steps), rtol=0, atol=1e-10)


def test_near_an_orthogonal_factor_and_transposition():
    g = np.random.default_rng(1).normal(0, 1, (16, 40))
    s = np.linalg.svd(newton_schulz(g), compute_uv=False)
    assert 0.65 < s.min() and s.max() < 1.25
    np.testing.assert_allclose(newton_schulz(g.T), newton_schulz(g).T, rtol=0, atol=1e-12)
    assert (newton_schulz(np.zeros((3, 4))) == 0).all()


def test_step():
    g = np.random.default_rng(2)
    p, grad, m = (g.normal(0, 1, (5, 8)) for _ in range(3))
    p1, m1, o = muon_step(p, grad, m, 0.1, momentum=0.0, weight_decay=0.5, rms=0.3)
    assert (m1 == grad).all()
    np.testing.assert_allclose(p1, 0.95 * p - 0.1 * 0.3 * np.sqrt(8) * newton_schulz(grad), rtol=1e-14)
    _, m1, o = muon_step(p, grad, m, 0.1, momentum=0.9, nesterov=False, grad_scale=2.0)
    np.testing.assert_allclose(m1, 0.9 * m + 0.2 * grad, rtol=1e-14)
    np.testing.assert_allclose(o, newton_schulz(m1), rtol=1e-12)
