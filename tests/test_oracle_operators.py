"""Pins of the oracle's operators: singular values, finite differences, torch.autograd, closed forms."""
import math

import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O


@pytest.mark.parametrize("shape,steps", [((5, 5), 5), ((4, 9), 5), ((9, 4), 3), ((1, 6), 1), ((1, 1), 5)])
def test_orthogonalize_maps_singular_values_by_the_polynomial(shape, steps):
    g = np.random.default_rng(1).standard_normal(shape)
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    s = s / (np.linalg.norm(g) + 1e-7)
    for _ in range(steps):
        a, b, c = O.NEWTON_SCHULZ
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(O.orthogonalize(g, steps), (u * s) @ vt, atol=1e-12)


def test_orthogonalize_of_zero_is_zero_and_transposes():
    assert not O.orthogonalize(np.zeros((3, 4))).any()
    g = np.random.default_rng(2).standard_normal((3, 7))
    assert np.allclose(O.orthogonalize(g.T), O.orthogonalize(g).T, atol=1e-13)


def test_muon_update_of_a_scaled_rotation():
    # an orthogonal gradient stays one: all singular values 1 / sqrt(n) go the same way
    q, _ = np.linalg.qr(np.random.default_rng(3).standard_normal((4, 4)))
    p, m = O.muon_update(np.ones((4, 4)), 3.0 * q, np.zeros((4, 4)), 0.1, 0.9, True, 0.5)
    s = 0.5
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    assert np.allclose(m, 3 * q) and np.allclose(p, 0.95 - 0.1 * 0.2 * 2 * s * q, atol=1e-6)


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_keeps_norms_and_depends_on_distances_alone(neighbours):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((6, 2, 10))
    pos = rng.integers(-50, 50, (6, 2))
    ang = O.rotary_angles(pos, [2, 2], 100.0)
    assert ang.shape == (6, 4) and np.allclose(ang[:, 1], pos[:, 0] / 10) and np.allclose(ang[:, 2], pos[:, 1])
    y = O.rotate(x, ang, neighbours)
    assert np.allclose(y[..., 8:], x[..., 8:]) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    far = O.rotate(x, O.rotary_angles(pos + np.array([7, -3]), [2, 2], 100.0), neighbours)
    dots = lambda v: np.einsum("ahd,bhd->abh", v, v)
    assert np.allclose(dots(y), dots(far))
    z = (x[0, 0, 0] + 1j * x[0, 0, 1]) if neighbours else (x[0, 0, 0] + 1j * x[0, 0, 4])
    w = z * np.exp(1j * ang[0, 0])
    assert np.isclose(y[0, 0, 0], w.real) and np.isclose(y[0, 0, 1 if neighbours else 4], w.imag)


def test_rms_norm_against_autograd():
    rng = np.random.default_rng(5)
    x, g, dy = rng.standard_normal((3, 4, 6)), rng.standard_normal(6), rng.standard_normal((3, 4, 6))
    xt, gt = torch.tensor(x, requires_grad=True), torch.tensor(g, requires_grad=True)
    yt = xt / torch.sqrt((xt ** 2).mean(-1, keepdim=True) + 1e-3) * gt
    yt.backward(torch.tensor(dy))
    y, cache = O.rms_norm_fwd(x, g, 1e-3)
    dx, dg = O.rms_norm_bwd(dy, cache, g)
    assert np.allclose(y, yt.detach().numpy()) and np.allclose(dx, xt.grad.numpy()) and np.allclose(dg, gt.grad.numpy())
