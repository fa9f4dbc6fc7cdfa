"""Gradients of linear layers on rows of 8 bits at the ends of their ranges: dX of more elements than one product addresses, dY that is infinite, NaN,
the largest there is, or so small that terms of it fall under bf16's least."""
import numpy as np
import pytest
import torch

from paper_2411_12780_amd import binding as P
from rows_helper import DEV, HALF, stream
from test_gpu_byte_linear import TYPES, ULP, Layer, check_backward, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("want,way", [(("dx",), None), (("dx",), 2), (("dx", "dw", "db"), 2), (("dx", "dw", "db"), None)])
def test_dx_in_stretches_of_rows(want, way):
    # 8400 rows 33288 elements apart: 2^28 of them and more from the first to the last of dX, two products
    check_backward(Layer(8400, 520, 264, torch.bfloat16, seed=11, room=32768), True, want, way=way)


def test_dx_of_rows_too_far_apart_for_stretches():
    check_backward(Layer(600, 136, 72, torch.bfloat16, seed=12, room=(1 << 19) + 8), True, ("dx",))


def test_dx_of_many_narrow_rows():
    m, k, n = 5000000, 64, 64
    gen = torch.Generator(device=DEV).manual_seed(13)
    dy, gate = (torch.randn(m, c, generator=gen, device=DEV).bfloat16() for c in (n, k))
    q, e = torch.randint(-127, 128, (n, k), generator=gen, device=DEV, dtype=torch.int8), torch.randint(-12, -6, (n,), generator=gen, device=DEV, dtype=torch.int8)
    cfg, dx = P.byte_linear_config(P.BF16, m, k, n), torch.empty(m, k, device=DEV, dtype=torch.bfloat16)
    ws = torch.empty(P.ppll_byte_linear_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    P.ppll_byte_linear_backward(cfg, None, P.byte_rows(q, e), P.rows(dy), P.rows(gate), P.rows(dx), None, None, ws, ws.numel(), stream())
    w = q.double() * torch.exp2(e.double())[:, None]
    for r in range(0, m, 1 << 20):
        d, g = dy[r:r + (1 << 20)].double(), gate[r:r + (1 << 20)].double()
        want, allowed = (d @ w) * g, ((n + 2) * 2 * ULP * (d.abs() @ w.abs()) + ULP * (d @ w).abs()) * g.abs()
        assert bool(((dx[r:r + (1 << 20)].double() - want).abs() <= allowed + 2.0 ** -8 * (want.abs() + allowed)).all()), r


def gradients(l, dy, want=("dx", "dw", "db")):
    m, k, n = l.shape
    dx, dw, db = l.empty(m, k), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
    size = P.ppll_byte_linear_workspace_bytes(l.cfg())
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
    P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx) if "dx" in want else None, dw if "dw" in want else None,
                                db if "db" in want else None, ws, size, stream())
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    return [dx.host() if "dx" in want else None, host(dw) if "dw" in want else None, host(db) if "db" in want else None]


def expected(l, dy):
    """The gradients and what their sums may be off by, in 64 bits: three terms of each of K elements, 2^-23 of the sum of magnitudes for an addition."""
    m, _, n = l.shape
    x, w = l.values()
    d = dy.host()
    with np.errstate(all="ignore"):
        finite = np.where(np.isfinite(d), d, 0)
        return [(d @ w, (n + 2) * 2 * ULP * (np.abs(finite) @ np.abs(w))), (x.T @ d, (m + 2) * 2 * ULP * (np.abs(x).T @ np.abs(finite))),
                (d.sum(0), (m + 2) * ULP * np.abs(finite).sum(0))]


def agree(got, want, allowed, half):
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), (got[odd], want[odd])
    got, want, allowed = got[~odd], want[~odd], allowed[~odd]
    assert (np.abs(got - want) <= allowed + half * (np.abs(want) + allowed)).all()


SIZES = [(70, 40, 24), (33, 21, 7), (300, 70, 333), (40, 64, 1200), (2500, 24, 72)]


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("want", [("dx", "dw", "db"), ("dx",)])
def test_infinite_gradients(precision, dtype, size, want):
    l = Layer(*size, dtype, seed=21)
    m, _, n = size
    dy = l.put(m, n)
    dy.view[3, 5], dy.view[m - 1, n - 1], dy.view[7, 0] = np.inf, -np.inf, np.inf
    for got, (ref, allowed), half in zip(gradients(l, dy, want), expected(l, dy), (HALF[dtype], 0, 0)):
        if got is not None:
            assert not np.isfinite(ref).all() and np.isfinite(ref).any()
            agree(got, ref, allowed, half)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_gradients_that_are_nan(precision, dtype, size):
    # of every kind: quiet, and with the lowest bit of the fraction alone
    l = Layer(*size, dtype, seed=22)
    m, _, n = size
    dy = l.put(m, n)
    bits, (quiet, least) = (torch.int32, (0x7fc00000, 0x7f800001)) if dtype == torch.float32 else (torch.int16, (0x7fc0, 0x7f81))
    dy.view.view(bits)[3, 5], dy.view.view(bits)[m - 1, n - 1] = quiet, least
    for got, (ref, allowed), half in zip(gradients(l, dy), expected(l, dy), (HALF[dtype], 0, 0)):
        assert np.isnan(ref).any() and np.isfinite(ref).any()
        agree(got, ref, allowed, half)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_the_largest_gradients(precision, dtype, size):
    # up to 127 * 2^-9 and 2^-6 of a value by which dY is multiplied, one of the largest a row and a column: no sum reaches infinity
    l = Layer(*size, dtype, seed=23)
    m, _, n = size
    l.ex[:] = -13
    l.x.exps[:m] = -13
    dy = l.put(m, n)
    most = torch.finfo(dtype).max
    dy.view[3, 5], dy.view[m - 1, n - 1], dy.view[7, 0] = most, -most, 0.998 * most
    for got, (ref, allowed), half in zip(gradients(l, dy), expected(l, dy), (HALF[dtype], 0, 0)):
        assert 1e35 < np.abs(ref).max() <= torch.finfo(dtype).max       # (a column sum of `most` and some small ones is `most`, in 64 bits too)
        agree(got, ref, allowed, half)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("scale", [2.0 ** -108, 1e-36])
def test_the_smallest_gradients(size, scale):
    # the third term of dY is off by half of bf16's least step, 2^-134, where dY is under 2^-110; sums in fp32 by its least step for each product
    l = Layer(*size, torch.float32, seed=24)
    m, k, n = size
    dy = l.put(m, n, scale=scale)
    x, w = l.values()
    least = [2.0 ** -134 * np.abs(w).sum(0)[None, :] + 3 * n * 2.0 ** -149, 2.0 ** -134 * np.abs(x).sum(0)[:, None] + 3 * m * 2.0 ** -149, m * 2.0 ** -149]
    for got, (ref, allowed), more in zip(gradients(l, dy), expected(l, dy), least):
        assert (np.abs(got - ref) <= allowed + more).all()
