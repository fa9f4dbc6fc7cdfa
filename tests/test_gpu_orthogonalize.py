"""Newton-Schulz orthogonalisation and the Muon step against the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(groups):
    # not a round number of bytes too many, and full of NaN: what a kernel reads it has written
    n = P.ppll_orthogonalize_workspace_bytes(groups)
    return torch.full((max(n, 16),), 255, dtype=torch.uint8, device=DEV)


def bound(g, steps):
    """Largest relative error (2-norm) that rounding at fp32 precision can leave.  A product of k terms whose operands carry 22 bits is off
    by at most d = 2^-21 (the two operands) + 2^-22 (the term left out) + k 2^-24 (sums) of the product of the norms of its operands, each
    rounding being at most half a step; a step of the iteration makes three of them, a X + b A X + c A A X with |A| <= 1.45 in the spectral
    norm: d (3 + |b| 1.45 * 2 + c 2.1 * 3) |X| at most, with the a X rounded as well under 31 d |X|.  What a step gets wrong grows by at most
    3.4445 (the largest slope of the polynomial, at 0) in each of the steps behind it.  The sum over k of the accumulation is taken as
    sqrt(k): its roundings have either sign (8 standard deviations of slack are in the 31 against 10 for random operands)."""
    x = g / (np.linalg.norm(g) + 1e-7)
    if x.shape[0] > x.shape[1]:
        x = x.T
    m, n = x.shape
    d = 2.0 ** -21 + 2.0 ** -22 + math.sqrt(n) * 2.0 ** -24
    err = 2.0 ** -22 * np.linalg.norm(x)
    for k in range(steps):
        err = 3.4445 * err + 31 * d * np.linalg.norm(x)
        x = one_step(x)
    return err / max(np.linalg.norm(x), 1e-300)


def one_step(x):
    a, b, c = O.NEWTON_SCHULZ
    s = x @ x.T
    return a * x + (b * s + c * s @ s) @ x


def matrices(blob, g):
    for i in range(g.count):
        yield np.lib.stride_tricks.as_strided(blob[g.offset + i * g.stride:], (g.rows, g.cols), (blob.itemsize * g.ld, blob.itemsize))


def blob_size(groups):
    return max(g.offset + max(g.count - 1, 0) * g.stride + (g.rows - 1) * g.ld + g.cols for g in groups)


def run(groups, values, dtype=torch.float32, steps=5, in_place=False):
    x = torch.from_numpy(values).to(DEV, dtype)
    out = x if in_place else torch.full_like(x, 7.0)
    before = x.clone()
    ws = workspace(groups)
    P.ppll_orthogonalize(groups, P.BF16 if dtype == torch.bfloat16 else P.FP32, steps, x, out, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(x.view(torch.uint8), before.view(torch.uint8))      # bits: NaN is NaN
    return before.double().cpu().numpy(), out.double().cpu().numpy()


def check(groups, given, got, steps=5, dtype=torch.float32, rest=7.0):
    touched = np.zeros(got.shape, dtype=bool)
    for g in groups:
        for a, b, t in zip(matrices(given, g), matrices(got, g), matrices(touched, g)):
            want = O.orthogonalize(a, steps)
            tol = bound(a, steps) + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
            norm, off = np.linalg.norm(want), np.linalg.norm(b - want)
            assert off <= tol * norm, (g.rows, g.cols, off / norm, tol)
            t[...] = True
    if rest is not None:
        assert (got[~touched] == rest).all()


SIZES = [(1, 1), (1, 7), (7, 1), (2, 3), (16, 16), (31, 33), (64, 64), (64, 128), (65, 63), (128, 64), (200, 40), (288, 32), (130, 257), (384, 384), (96, 1000),
         (1000, 96), (1, 8192), (8192, 2), (576, 64), (27, 16)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, dtype):
    groups = [P.matrix_group(0, rows, cols, count=3)]
    values = np.random.default_rng(rows * 10007 + cols).standard_normal(3 * rows * cols).astype(np.float32)
    given, got = run(groups, values, dtype)
    check(groups, given, got, dtype=dtype)


@pytest.mark.parametrize("steps", [1, 2, 5, 8])
def test_steps(steps):
    groups = [P.matrix_group(0, 48, 80, count=2), P.matrix_group(2 * 48 * 80, 150, 70)]
    values = np.random.default_rng(steps).standard_normal(blob_size(groups)).astype(np.float32)
    given, got = run(groups, values, steps=steps)
    check(groups, given, got, steps)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layouts(dtype, in_place):
    # parts of a wide weight in three layers, rows with room behind them, odd offsets, matrices far apart, an empty group
    groups = [P.matrix_group(5 + i * 40, 40, 40, ld=123, count=3, stride=9001) for i in range(3)]
    groups += [P.matrix_group(5 + 40 * 123, 17, 90, ld=91, count=3, stride=9001), P.matrix_group(40000, 33, 9, ld=50, count=4, stride=11),
               P.matrix_group(50000, 5, 5, count=0), P.matrix_group(60001, 140, 200, ld=201, count=2, stride=50003)]
    values = np.random.default_rng(11).standard_normal(blob_size(groups) + 13).astype(np.float32)
    if in_place:
        values[-13:] = 7.0
    given, got = run(groups, values, dtype, in_place=in_place)
    check(groups, given, got, dtype=dtype, rest=None if in_place else 7.0)
    if in_place:
        touched = np.zeros(got.shape, dtype=bool)
        for g in groups:
            for t in matrices(touched, g):
                t[...] = True
        assert np.array_equal(got[~touched], given[~touched])


def test_many_matrices_and_large_tiles():
    # enough tiles of 128 for the larger kernel; sizes that are no multiple of it
    groups = [P.matrix_group(0, 300, 420, count=30), P.matrix_group(30 * 300 * 420, 700, 260, count=20), P.matrix_group(30 * 300 * 420 + 20 * 700 * 260, 9, 4)]
    values = np.random.default_rng(12).standard_normal(blob_size(groups)).astype(np.float32)
    given, got = run(groups, values)
    check(groups, given, got)


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1e-3, 1e18, 1e30])
def test_scales(scale):
    # norms whose squares are out of the range of 32 bits; under 1e-7 the added constant takes over
    groups = [P.matrix_group(0, 24, 40, count=2), P.matrix_group(1920, 100, 100)]
    values = (np.random.default_rng(13).standard_normal(blob_size(groups)) * scale).astype(np.float32)
    given, got = run(groups, values)
    for g in groups:
        for a, b in zip(matrices(given, g), matrices(got, g)):
            want = O.orthogonalize(a)
            off, most = np.linalg.norm(b - want), bound(a / np.abs(a).max(), 5) * np.linalg.norm(want) + 1e-25
            assert off <= most


def test_spectra():
    # low rank beside noise, a spectrum over four decades, exact rank 1, one huge row
    rng = np.random.default_rng(14)
    m, n = 120, 180
    low = rng.standard_normal((m, 4)) @ rng.standard_normal((4, n)) + 0.01 * rng.standard_normal((m, n))
    u, _, vt = np.linalg.svd(rng.standard_normal((m, n)), full_matrices=False)
    rank1 = np.outer(rng.standard_normal(m), rng.standard_normal(n))
    huge = rng.standard_normal((m, n))
    huge[3] *= 1e4
    values = np.stack([low, (u * np.logspace(0, -4, m)) @ vt, rank1, huge]).astype(np.float32).reshape(-1)
    groups = [P.matrix_group(0, m, n, count=4)]
    given, got = run(groups, values)
    check(groups, given, got)


@pytest.mark.parametrize("rows,cols", [(20, 30), (130, 200)])
def test_zeros_and_values_that_are_not_finite_stay_in_their_matrix(rows, cols):
    groups = [P.matrix_group(0, rows, cols, count=4)]
    values = np.random.default_rng(15).standard_normal((4, rows, cols)).astype(np.float32)
    values[0] = 0
    values[1, 3, 5] = np.nan
    values[2, rows - 1, 0] = np.inf
    given, got = run(groups, values.reshape(-1))
    got = got.reshape(4, rows, cols)
    assert (got[0] == 0).all() and np.isnan(got[1]).all() and np.isnan(got[2]).all()
    want, last = O.orthogonalize(given.reshape(4, rows, cols)[3]), given.reshape(4, rows, cols)[3]
    off, most = np.linalg.norm(got[3] - want), bound(last, 5) * np.linalg.norm(want)
    assert off <= most


def muon(groups, p, g, m, nesterov=True, shadow=True, calls=1, lr=0.02, momentum=0.9, decay=0.1, steps=5):
    t = [torch.from_numpy(v).to(DEV) for v in (p, g, m)]
    s = torch.full((p.size,), 3.0, dtype=torch.bfloat16, device=DEV) if shadow else None
    ws = workspace(groups)
    for _ in range(calls):
        P.ppll_muon_step(groups, steps, t[1], t[2], t[0], s, lr, momentum, nesterov, decay, ws, ws.numel(), stream())
    torch.cuda.synchronize()
    assert np.array_equal(t[1].cpu().numpy(), g)
    return t[0].cpu().numpy(), t[2].cpu().numpy(), s


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("dim,mlp,layers", [(16, 40, 2), (64, 128, 2), (72, 100, 1), (136, 300, 2)])
def test_muon_step(dim, mlp, layers, nesterov):
    layer = 4 * dim * dim + 2 * dim * mlp + 3
    groups = [P.matrix_group(1 + i * dim, dim, dim, ld=3 * dim, count=layers, stride=layer) for i in range(3)]
    groups += [P.matrix_group(1 + 3 * dim * dim, dim, dim, count=layers, stride=layer), P.matrix_group(1 + 4 * dim * dim, dim, mlp, count=layers, stride=layer),
               P.matrix_group(1 + 4 * dim * dim + dim * mlp, mlp, dim, count=layers, stride=layer)]
    rng = np.random.default_rng(dim)
    n = layer * layers + 1
    p, g, m = (0.02 * rng.standard_normal(n)).astype(np.float32), rng.standard_normal(n).astype(np.float32), (2 * rng.standard_normal(n)).astype(np.float32)
    lr, mu, wd = 0.02, 0.9, 0.1
    got_p, got_m, shadow = muon(groups, p, g, m, nesterov, lr=lr, momentum=mu, decay=wd, calls=2)
    assert np.array_equal(shadow.float().cpu().numpy()[1:1 + 3], torch.from_numpy(got_p).bfloat16().float().numpy()[1:1 + 3])
    touched = np.zeros(n, dtype=bool)
    for group in groups:
        for P0, G, M, gp, gm, t in zip(*(matrices(v, group) for v in (p, g, m, got_p, got_m, touched))):
            wp, wm = P0.astype(np.float64), M.astype(np.float64)
            err = 0.0
            for _ in range(2):
                wp, wm = O.muon_update(wp, G.astype(np.float64), wm, lr, mu, nesterov, wd)
                u = G + mu * wm if nesterov else wm
                # the update's own error (its momentum is rounded to fp32 as well), and p rounded twice
                err += lr * 0.2 * math.sqrt(max(G.shape)) * (bound(u, 5) * np.linalg.norm(O.orthogonalize(u))) + 2 ** -23 * np.linalg.norm(wp)
            off = np.linalg.norm(gp - wp)
            assert off <= err
            # two fused operations with one rounding each
            assert np.abs(gm - wm).max() <= 2 * 2 ** -24 * (np.abs(wm).max() + np.abs(M).max())
            t[...] = True
    s = shadow.float().cpu().numpy()
    assert np.array_equal(got_p[~touched], p[~touched]) and np.array_equal(got_m[~touched], m[~touched]) and (s[~touched] == 3).all()
    assert np.array_equal(s[touched], torch.from_numpy(got_p[touched]).bfloat16().float().numpy())


def test_muon_without_shadow_momentum_or_decay():
    groups = [P.matrix_group(0, 30, 50)]
    rng = np.random.default_rng(20)
    p, g, m = (rng.standard_normal(1500).astype(np.float32) for _ in range(3))
    got_p, got_m, _ = muon(groups, p, g, m, shadow=False, momentum=0.0, decay=0.0, lr=0.5)
    assert np.array_equal(got_m, g)
    want = p.astype(np.float64) - 0.1 * math.sqrt(50) * O.orthogonalize(g.astype(np.float64).reshape(30, 50)).reshape(-1)
    off, size = np.linalg.norm(got_p - want), np.linalg.norm(O.orthogonalize(g.astype(np.float64).reshape(30, 50)))
    most = 0.1 * math.sqrt(50) * bound(g.reshape(30, 50).astype(np.float64), 5) * size + 2 ** -23 * np.linalg.norm(want)
    assert off <= most


def test_results_do_not_depend_on_company_or_repetition():
    # bits of a matrix are the same alone and among others of its kernel, and on every call
    rng = np.random.default_rng(21)
    values = rng.standard_normal(20 * 48 * 60).astype(np.float32)
    _, many = run([P.matrix_group(0, 48, 60, count=20)], values)
    _, again = run([P.matrix_group(0, 48, 60, count=20)], values)
    _, one = run([P.matrix_group(7 * 2880, 48, 60)], values)
    assert np.array_equal(many, again) and np.array_equal(many[7 * 2880:8 * 2880], one[7 * 2880:8 * 2880])


@pytest.mark.parametrize("rows,cols", [(40, 60), (150, 260)])
def test_captured_and_replayed_on_another_stream(rows, cols):
    groups = [P.matrix_group(0, rows, cols, count=3)]
    rng = np.random.default_rng(22)
    n = 3 * rows * cols
    g, p0 = (torch.from_numpy(rng.standard_normal(n).astype(np.float32)).to(DEV) for _ in range(2))
    ws = workspace(groups)
    p, m = p0.clone(), torch.zeros_like(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        P.ppll_muon_step(groups, 5, g, m, p, None, 0.1, 0.9, True, 0.01, ws, ws.numel(), stream())
    eager_p, eager_m, other = p0.clone(), torch.zeros_like(g), workspace(groups)
    p.copy_(p0)
    m.zero_()
    for k in range(3):
        g.copy_(torch.from_numpy(rng.standard_normal(n).astype(np.float32)))
        graph.replay()
        P.ppll_muon_step(groups, 5, g, eager_m, eager_p, None, 0.1, 0.9, True, 0.01, other, other.numel(), stream())
        torch.cuda.synchronize()
        assert torch.equal(p, eager_p) and torch.equal(m, eager_m), k


def test_two_calls_at_once_on_two_streams():
    groups = [P.matrix_group(0, 200, 300, count=4)]
    rng = np.random.default_rng(23)
    xs = [torch.from_numpy(rng.standard_normal(4 * 60000).astype(np.float32)).to(DEV) for _ in range(2)]
    alone = []
    for x in xs:
        out, ws = torch.empty_like(x), workspace(groups)
        P.ppll_orthogonalize(groups, P.FP32, 5, x, out, ws, ws.numel(), stream())
        torch.cuda.synchronize()
        alone.append(out)
    outs, wss, streams = [torch.empty_like(x) for x in xs], [workspace(groups) for _ in xs], [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for x, out, ws, s in zip(xs, outs, wss, streams):
        P.ppll_orthogonalize(groups, P.FP32, 5, x, out, ws, ws.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_no_element_of_many_loses_its_low_term():
    # 400 matrices whose every element passes through both conversions of an operand some ten times; fp32 arithmetic leaves 1e-6 of each
    groups = [P.matrix_group(0, 64, 64, count=400)]
    values = np.random.default_rng(24).standard_normal(400 * 4096).astype(np.float32)
    given, got = run(groups, values)
    x = torch.from_numpy(given.reshape(400, 64, 64))
    x, y = (x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)).double(), (x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)).float()
    a, b, c = O.NEWTON_SCHULZ
    for _ in range(5):
        x, y = (v * a + (b * v @ v.transpose(1, 2) + c * (v @ v.transpose(1, 2)) @ (v @ v.transpose(1, 2))) @ v for v in (x, y))
    off = lambda v: ((v.double() - x).norm(dim=(1, 2)) / x.norm(dim=(1, 2))).max().item()  # noqa: E731
    own, fp32 = off(torch.from_numpy(got.reshape(400, 64, 64))), off(y)
    assert own <= 2 * fp32, (own, fp32)


@pytest.mark.parametrize("rows,cols", [(64, 500), (33, 1000), (100, 250), (128, 144), (129, 129), (128, 160), (160, 96), (16, 2000), (32, 1264), (32, 1300), (64, 64)])
def test_sizes_on_both_sides_of_what_one_workgroup_holds(rows, cols):
    for shape in ((rows, cols), (cols, rows)):
        groups = [P.matrix_group(3, *shape, ld=shape[1] + 1, count=2)]
        values = np.random.default_rng(rows + cols).standard_normal(blob_size(groups)).astype(np.float32)
        given, got = run(groups, values)
        check(groups, given, got)


# few tiles and long rows: the k of a tile is in pieces, whose sums one of its workgroups adds up; with 1536 x 3000 in the larger tiles
@pytest.mark.parametrize("rows,cols,count", [(256, 2048, 1), (130, 2001, 2), (4000, 65, 1), (520, 1990, 1), (1000, 1000, 1), (1536, 3000, 1)])
def test_few_tiles_of_long_rows(rows, cols, count):
    groups = [P.matrix_group(0, rows, cols, count=count)]
    values = np.random.default_rng(rows + cols).standard_normal(count * rows * cols).astype(np.float32)
    given, got = run(groups, values, steps=2)
    check(groups, given, got, steps=2)
    for _ in range(6):                                      # whichever piece comes last: the same bits
        assert np.array_equal(run(groups, values, steps=2)[1], got)


def test_pieces_replayed_with_calls_between():
    groups = [P.matrix_group(0, 200, 2048), P.matrix_group(200 * 2048, 2048, 140)]
    x = torch.randn(blob_size(groups), device=DEV)
    out, eager = torch.empty_like(x), torch.empty_like(x)
    ws = workspace(groups)
    s = torch.cuda.Stream()
    call = lambda dst: P.ppll_orthogonalize(groups, P.FP32, 5, x, dst, ws, ws.numel(), stream())  # noqa: E731
    call(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(out)
    for _ in range(4):
        x.copy_(torch.randn_like(x))
        ws.fill_(255)                                       # nothing is kept in the workspace from call to call
        graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
