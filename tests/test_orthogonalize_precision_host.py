"""That the limits of test_gpu_orthogonalize_precision.py see a term that is missing: an emulation of the products in numpy, whole and with parts left out."""
import numpy as np
import pytest

from oracle import ppll_oracle as O

ALLOWED = 3


def split(v, low):
    v = np.float32(16384) * v.astype(np.float32)
    hi = v.astype(np.float16)
    return hi.astype(np.float32), ((v - hi.astype(np.float32)) * np.float32(low)).astype(np.float16).astype(np.float32)


def product(p, q, low, left_out):
    """P Q' of operands in two terms; left_out: 0 nothing, 1 a cross term, 2 both"""
    cross = p[0] @ q[1].T if left_out < 2 else np.float32(0)
    if left_out < 1:
        cross = cross + p[1] @ q[0].T
    return (p[0] @ q[0].T + cross / np.float32(low)) / np.float32(2 ** 28)


def emulated(u, steps=5, low=2048, left_out=0, low_terms=True):
    a, b, c = (np.float32(v) for v in O.NEWTON_SCHULZ)
    terms = lambda v: split(v, low) if low_terms else (split(v, low)[0], np.zeros(v.shape, np.float32))  # noqa: E731
    value = lambda t: (t[0] + t[1] / np.float32(low)) / np.float32(16384)  # noqa: E731
    turned = lambda t: (t[0].T, t[1].T)  # noqa: E731
    x = terms((u / np.linalg.norm(u)).astype(np.float32))
    for _ in range(steps):
        s = terms(product(x, x, low, left_out))
        poly = terms(b * value(s) + c * product(s, s, low, left_out))
        result = a * value(x) + product(poly, turned(x), low, left_out)
        x = terms(result)
    return result


def iterate(u, dtype, steps=5):
    a, b, c = (dtype(v) for v in O.NEWTON_SCHULZ)
    x = (u / np.linalg.norm(u)).astype(dtype)
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return x


def off(x, want, axis=None):
    return np.max(np.linalg.norm(x - want, axis=axis) / np.linalg.norm(want, axis=axis))


@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("rows,cols", [(32, 288), (64, 64), (201, 333), (256, 2048), (384, 384)])
def test_a_missing_term_is_seen(rows, cols, steps):
    u = np.random.default_rng([rows, cols]).standard_normal((rows, cols)).astype(np.float32).astype(np.float64)
    want = iterate(u, np.float64, steps)
    limit = ALLOWED * off(iterate(u, np.float32, steps), want)
    assert off(emulated(u, steps), want) <= limit
    assert off(emulated(u, steps, left_out=1), want) > 2 * limit
    assert off(emulated(u, steps, left_out=2), want) > 2 * limit
    assert off(emulated(u, steps, low_terms=False), want) > 2 * limit


def test_low_terms_at_the_scale_of_the_high_ones_lose_small_rows():
    u = np.random.default_rng(3).standard_normal((96, 400))
    u[:4] *= 1e-4
    u[4:8] *= 1e-6
    u = u.astype(np.float32).astype(np.float64)
    want, fp32 = iterate(u, np.float64), iterate(u, np.float32)
    for rows, size in ((slice(0, 4), 1e-4), (slice(4, 8), 1e-6)):
        limit = ALLOWED * off(fp32[rows], want[rows], 1) + 3 * 1.41 * 2.0 ** -50 * (96 * 400) ** 0.5 / size
        assert off(emulated(u)[rows], want[rows], 1) <= limit
        assert off(emulated(u, low=1)[rows], want[rows], 1) > 2 * limit
