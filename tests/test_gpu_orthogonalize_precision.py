"""The precision of Newton-Schulz orthogonalisation: beside 64 bits, its errors are held against those of the same iteration in fp32.

An operand is two fp16 terms of 11 bits each, so what is stored is off by at most 2^-22 and by about as much as a rounding to fp32 in the mean; the product
of two low terms that is left out is of that size as well, and the sums are sums of fp32.  Three errors of the size of fp32's one, of either sign: under
twice its error for random matrices, and `FP32` times is allowed.  What is left out of a product by mistake - one of the cross terms, the low terms - costs
2^-12 of it (test_orthogonalize_precision_host.py shows that on an emulation)."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP32 = 3
FLOOR = 2.0 ** -50          # of a matrix of norm 1: half the last place of a low term


def stream():
    return torch.cuda.current_stream().cuda_stream


def start_of(u):
    u = u.double()
    return u / (u.norm() + 1e-7)


def iterate(x, steps):
    a, b, c = O.NEWTON_SCHULZ
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t().contiguous() if tall else x


def both(u, steps):
    """The definition in 64 bits, and the same products in 32."""
    return iterate(start_of(u), steps), iterate(start_of(u).float(), steps).double()


def call(groups, x, steps=5):
    out, n = torch.full_like(x, 7.0), P.ppll_orthogonalize_workspace_bytes(groups)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    P.ppll_orthogonalize(groups, P.FP32, steps, x, out, ws, n, stream())
    torch.cuda.synchronize()
    return out


def off(got, want, dim=None):
    norm = torch.linalg.vector_norm
    return (norm(got.double() - want, dim=dim) / norm(want, dim=dim)).max().item()


# one workgroup a matrix; tiles of 64 and of 128, wide and tall, whole and with the k in pieces
SIZES = [(64, 64, 3), (288, 32, 3), (120, 100, 2), (201, 333, 5), (333, 201, 5), (384, 384, 16), (256, 2048, 1), (2001, 130, 2), (1536, 2000, 2), (1100, 700, 12),
         (520, 1990, 1), (1024, 1024, 8)]


@pytest.mark.parametrize("steps", [1, 5])
@pytest.mark.parametrize("rows,cols,count", SIZES)
def test_errors_are_those_of_fp32(rows, cols, count, steps):
    x = torch.from_numpy(np.random.default_rng([rows, cols]).standard_normal((count, rows, cols)).astype(np.float32)).to(DEV)
    got = call([P.matrix_group(0, rows, cols, count=count)], x, steps)
    worst = [0.0, 0.0]
    for u, v in zip(x[:3], got[:3]):
        want, fp32 = both(u, steps)
        worst = [max(worst[0], off(v, want)), max(worst[1], off(fp32, want))]
    assert worst[0] <= FP32 * worst[1], worst


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("rows,cols,count", [(64, 128, 4), (384, 384, 16), (384, 1536, 8), (1536, 384, 8), (200, 2000, 1)])
def test_errors_of_a_muon_step_are_those_of_fp32(rows, cols, count, nesterov):
    # parameters of 0 without decay: what is left is the update
    rng = np.random.default_rng([rows, cols, 1])
    g, m = (torch.from_numpy(rng.standard_normal((count, rows, cols)).astype(np.float32)).to(DEV) for _ in range(2))
    groups, p, lr, mu = [P.matrix_group(0, rows, cols, count=count)], torch.zeros_like(g), 0.5, 0.9
    n = P.ppll_orthogonalize_workspace_bytes(groups)
    ws = torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)
    momenta = m.clone()
    P.ppll_muon_step(groups, 5, g, momenta, p, None, lr, mu, nesterov, 0.0, ws, n, stream())
    torch.cuda.synchronize()
    worst = [0.0, 0.0]
    scale = -lr * 0.2 * max(rows, cols) ** 0.5
    for k in range(min(count, 3)):
        def update(m, g):
            m = np.float32(mu).item() * m + g
            return np.float32(mu).item() * m + g if nesterov else m
        want = iterate(start_of(update(m[k].double(), g[k].double())), 5) * scale
        fp32 = iterate(start_of(update(m[k], g[k])).float(), 5).double() * scale
        worst = [max(worst[0], off(p[k], want)), max(worst[1], off(fp32, want))]
    assert worst[0] <= FP32 * worst[1], worst


@pytest.mark.parametrize("across", [False, True])
@pytest.mark.parametrize("rows,cols", [(64, 64), (96, 120), (256, 1024), (700, 300), (384, 384)])
def test_rows_and_columns_far_under_the_others_keep_their_digits(rows, cols, across):
    # every product is linear in a row (a column) of X, so fp32 arithmetic leaves a small one the digits that it leaves a large one.  A row of size s beside
    # others of 1 has elements of s / sqrt(rows cols), and each is stored to FLOOR; a step makes it 3.4445 times as large, so what the first ones lost
    # counts most: 1 + 1 / 3.4445 + .. = 1.41 times it, three times for the three products
    rng = np.random.default_rng([rows, cols, 2])
    small = {1e-2: range(4), 1e-4: range(4, 8), 1e-6: range(8, 12)}
    values = rng.standard_normal((rows, cols))
    for size, lines in small.items():
        for k in lines:
            (values.T if across else values)[k] *= size
    x = torch.from_numpy(values.astype(np.float32)).to(DEV)
    got = call([P.matrix_group(0, rows, cols)], x)
    want, fp32 = both(x, 5)
    for size, lines in small.items():
        lines = list(lines)
        part = (lambda t: t[:, lines].t()) if across else (lambda t: t[lines])  # noqa: E731
        own, usual = off(part(got), part(want), 1), off(part(fp32), part(want), 1)
        assert own <= FP32 * usual + 3 * 1.41 * FLOOR * (rows * cols) ** 0.5 / size, (size, own, usual)


@pytest.mark.parametrize("steps", [1, 3, 5])
@pytest.mark.parametrize("norm", [1e-28, 1e-10, 1e-8, 3e-8, 1e-7, 1e-6, 1e-3, 1e20, 1e32])
def test_norms_about_the_constant_and_beyond_32_bits(norm, steps):
    # 1e-8: X begins at 0.09 and its norm passes 1 within the steps.  A few roundings of the factor that keeps the stored norm at 1 come on top: eight at most
    shapes = [(130, 200, 2), (300, 140, 1), (40, 30, 1)]
    groups, at, parts = [], 0, []
    rng = np.random.default_rng(steps)
    for rows, cols, count in shapes:
        groups.append(P.matrix_group(at, rows, cols, count=count))
        for _ in range(count):
            v = rng.standard_normal((rows, cols))
            parts.append((v / np.linalg.norm(v) * norm).astype(np.float32))
            at += rows * cols
    x = torch.from_numpy(np.concatenate([p.reshape(-1) for p in parts])).to(DEV)
    got, at = call(groups, x, steps), 0
    for p in parts:
        want, fp32 = both(torch.from_numpy(p).to(DEV), steps)
        own, usual = off(got[at:at + p.size].view(p.shape), want), off(fp32, want)
        assert own <= FP32 * usual + 8 * 2.0 ** -24, (p.shape, own, usual)
        at += p.size


def test_momenta_about_the_constant():
    # the same through the Muon step, whose norm is the momentum's
    rng = np.random.default_rng(9)
    for rows, cols in ((130, 200), (300, 140)):
        for norm in (1e-20, 1e-8, 1e-7):
            v = rng.standard_normal((rows, cols))
            g = torch.from_numpy((v / np.linalg.norm(v) * norm).astype(np.float32)).to(DEV)
            groups, p, m = [P.matrix_group(0, rows, cols)], torch.zeros_like(g), torch.zeros_like(g)
            n = P.ppll_orthogonalize_workspace_bytes(groups)
            ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)
            P.ppll_muon_step(groups, 5, g, m, p, None, 1.0, 0.9, False, 0.0, ws, n, stream())
            torch.cuda.synchronize()
            want, fp32 = (t * -0.2 * max(rows, cols) ** 0.5 for t in both(g, 5))
            assert torch.equal(m, g) and off(p, want) <= FP32 * off(fp32, want) + 8 * 2.0 ** -24, (rows, cols, norm)
