"""Group norm with an activation, forward and backward, against the float64 oracle.

Tolerances.  A sum over a group is a chain of 64 additions a thread and at most 20 levels above: 100 roundings of the mean magnitude.  Mean, squares about
it and what follows: under 300 roundings of the magnitudes that enter.  Sums over images add 64 chains of images / 64.  Activations: the normal CDF within
1e-6, the logistic function within 4e-6 (its exponential off by 2^-22 |z| in bf16's form), their slopes within 4 times that."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from rows_helper import DEV, HALF, Placed, PlacedBytes, stream

pytestmark = pytest.mark.gpu
TYPES = [(P.FP32, torch.float32), (P.BF16, torch.bfloat16)]
ACTS = {"none": P.ACT_NONE, "relu": P.ACT_RELU, "silu": P.ACT_SILU, "gelu": P.ACT_GELU}
ULP, EPS = 2.0 ** -24, 1e-5


def rows(p):
    return None if p is None else P.rows(p.view)


def device(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DEV)


class Case:
    def __init__(self, images, pixels, channels, groups, dtype, act="none", residual=False, room=0, shift=0, offset=0.5, seed=0):
        rng = np.random.default_rng([seed, images, pixels, channels, groups])
        self.__dict__.update({k: v for k, v in locals().items() if k not in ("self", "rng")})
        n = images * pixels
        self.place = dict(room=room, shift=shift)
        put = lambda a: Placed(torch.from_numpy(a.astype(np.float32)), dtype, **self.place)  # noqa: E731
        self.x = put(rng.standard_normal((n, channels)) + offset * rng.standard_normal((1, channels)))
        self.res = put(rng.standard_normal((n, channels))) if residual else None
        self.dy = put(1e-2 * rng.standard_normal((n, channels)))
        self.g, self.b = device(1 + 0.3 * rng.standard_normal(channels)), device(0.3 * rng.standard_normal(channels))
        self.cfg = P.group_norm_config(P.BF16 if dtype == torch.bfloat16 else P.FP32, images, pixels, channels, groups, ACTS[act], EPS)

    def empty(self):
        return Placed((self.images * self.pixels, self.channels), self.dtype, **self.place)

    def maps(self, a):
        return a.reshape(self.images, self.pixels, self.channels)

    def workspace(self):
        size = P.ppll_group_norm_workspace_bytes(self.cfg)
        ws = torch.full((max(size, 16) + 64,), 0x77, dtype=torch.uint8, device=DEV)
        return ws, size

    def forward(self, keep=None, y=None):
        y = y or self.empty()
        stats = torch.full((self.images, self.groups, 2), 7.0, device=DEV)
        ws, size = self.workspace()
        P.ppll_group_norm_forward(self.cfg, rows(self.x), self.g, self.b, rows(self.res), rows(y), stats,
                                  None if keep is None else P.byte_rows(keep.store, keep.exps), ws, size, stream())
        assert bool((ws[size:] == 0x77).all())
        return y, stats

    def oracle(self):
        res = None if self.res is None else self.maps(self.res.host())
        return O.group_norm_fwd(self.maps(self.x.host()), self.g.double().cpu().numpy(), self.b.double().cpu().numpy(), self.groups, EPS, self.act, res)


def act_room(act):
    return {"none": 0.0, "relu": 0.0, "silu": 4e-6, "gelu": 1e-6}[act]


def spread(c, per_group):
    """[images, groups] -> [images, 1, channels]"""
    return np.repeat(per_group, c.channels // c.groups, axis=1)[:, None, :]


def check_forward(c, kept=False):
    keep = PlacedBytes(c.images * c.pixels, c.channels, room=16) if kept else None
    y, stats = c.forward(keep)
    want, want_stats, z = c.oracle()
    x, g = np.abs(c.maps(c.x.host())), np.abs(c.g.double().cpu().numpy())
    mean_abs = spread(c, x.reshape(c.images, c.pixels, c.groups, -1).mean(axis=(1, 3)))
    r = spread(c, want_stats[..., 1])
    off_z = 300 * ULP * (g * r * (x + mean_abs) * (1 + mean_abs * r) + np.abs(c.b.double().cpu().numpy()) + np.abs(z))
    allowed = 1.2 * off_z + act_room(c.act) * (1 + np.abs(z))
    assert (np.abs(c.maps(y.host()) - want) <= allowed + HALF[c.dtype] * (np.abs(want) + allowed)).all()
    s, m0 = stats.double().cpu().numpy(), mean_abs.reshape(c.images, -1)[:, ::c.channels // c.groups]
    assert (np.abs(s[..., 0] - want_stats[..., 0]) <= 100 * ULP * m0 + ULP * np.abs(want_stats[..., 0])).all()
    # the variance is off by some 200 roundings of itself and by the mean's error squared
    assert (np.abs(s[..., 1] / want_stats[..., 1] - 1) <= 300 * ULP + (100 * ULP * m0 * want_stats[..., 1]) ** 2).all()
    assert y.untouched_around()
    if kept:
        q, e = O.byte_rows(c.x.host())
        assert np.array_equal(keep.q(), q) and np.array_equal(keep.e(), e) and keep.padding_is_zero_and_the_rest_untouched()


# every way that channels of a group lie in pieces of 8, images in one go, in slabs and in pieces
SHAPES = [(1, 1, 8, 1), (2, 1, 1, 1), (3, 5, 16, 4), (2, 7, 20, 4), (2, 9, 24, 3), (2, 30, 6, 6), (3, 64, 8, 4), (2, 100, 40, 8), (2, 33, 96, 32), (5, 49, 64, 8),
          (128, 64, 16, 4), (2, 1024, 16, 4), (2, 1000, 48, 2), (1, 3000, 64, 8), (2, 2500, 72, 9), (2, 5000, 21, 3), (1, 700, 512, 32), (1, 40, 4096, 16),
          (2, 300, 1100, 11), (1, 20000, 8, 8), (1, 9216, 64, 32), (300, 4, 32, 2), (2, 5, 1030, 103)]


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(precision, dtype, shape):
    if shape[1] * shape[2] // shape[3] > 1:
        check_forward(Case(*shape, dtype), kept=True)
    check_forward(Case(*shape, dtype, act="relu", residual=True))


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("place", [dict(), dict(room=1), dict(room=5, shift=3), dict(room=8, shift=8)])
def test_forward_activations_of_strided_maps(precision, dtype, act, place):
    for shape in ((3, 50, 24, 4), (1, 6000, 24, 6)):
        check_forward(Case(*shape, dtype, act=act, residual=True, seed=1, **place), kept=True)
        check_forward(Case(*shape, dtype, act=act, seed=1, **place))


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("shape", [(2, 50, 32, 4), (1, 9000, 64, 4)])
def test_a_mean_far_from_zero(precision, dtype, shape):
    check_forward(Case(*shape, dtype, offset=200.0, seed=2))


def test_forward_in_place():
    for shape in ((2, 50, 32, 4), (1, 9000, 40, 8)):
        c = Case(*shape, torch.bfloat16, act="relu", residual=True)
        y, _ = c.forward()
        c.forward(y=c.x)
        assert torch.equal(c.x.view, y.view)
        c = Case(*shape, torch.bfloat16, act="relu", residual=True)
        c.forward(y=c.res)
        assert torch.equal(c.res.view, y.view)


@pytest.mark.parametrize("shape", [(3, 20, 16, 2), (2, 9000, 40, 4)])
def test_a_nan_stays_in_its_group_of_its_image(shape):
    c = Case(*shape, torch.bfloat16, act="relu", residual=True)
    c.x.view[7, 1] = float("nan")
    y, stats = c.forward()
    nan = np.zeros(c.maps(y.host()).shape, dtype=bool)
    nan[0, :, :c.channels // c.groups] = True
    assert np.array_equal(np.isnan(c.maps(y.host())), nan)
    assert bool(stats[0, 0].isnan().all()) and bool(stats.reshape(-1)[2:].isfinite().all())


def check_backward(c, from_bytes=False, d_residual=True):
    y, stats = c.forward()
    x = c.maps(c.x.host())
    x8 = None
    if from_bytes:
        q, e = O.byte_rows(c.x.host())
        x8 = PlacedBytes(c.images * c.pixels, c.channels, q, e, room=16)
        x = c.maps(O.byte_values(q, e))
    dx, dres = c.empty(), c.empty() if d_residual else None
    dg, db = torch.full((c.channels,), 7.0, device=DEV), torch.full((c.channels,), 7.0, device=DEV)
    ws, size = c.workspace()
    P.ppll_group_norm_backward(c.cfg, None if from_bytes else rows(c.x), P.byte_rows(x8.store, x8.exps) if from_bytes else None, stats, c.g, c.b,
                               rows(c.res), rows(y), rows(c.dy), rows(dx), rows(dres), dg, db, ws, size, stream())
    assert bool((ws[size:] == 0x77).all())
    g, b, st = (t.double().cpu().numpy() for t in (c.g, c.b, stats))
    mean, r = spread(c, st[..., 0]), spread(c, st[..., 1])
    xhat = (x - mean) * r
    z = xhat * g + b + (0 if c.res is None else c.maps(c.res.host()))
    dy, half = c.maps(c.dy.host()), HALF[c.dtype]
    slope = (c.maps(y.host()) > 0).astype(float) if c.act == "relu" else O.activation(c.act, z)[1]
    dz = dy * slope
    off_x = 3 * ULP * (np.abs(x) + np.abs(mean)) * r
    off_dz = np.abs(dy) * (4 * act_room(c.act) * (1 + np.abs(z)) + (0 if c.act in ("none", "relu") else 2 * (off_x * np.abs(g) + 3 * ULP * np.abs(z)))) + ULP * np.abs(dz)
    if d_residual:
        assert (np.abs(c.maps(dres.host()) - dz) <= off_dz + half * (np.abs(dz) + off_dz)).all()
        assert dres.untouched_around()
    want, want_g, want_b = O.group_norm_bwd(dz, x, st, g)
    mean_of = lambda a: spread(c, a.reshape(c.images, c.pixels, c.groups, -1).mean(axis=(1, 3)))  # noqa: E731
    terms = np.abs(dz * g) + mean_of(np.abs(dz * g)) + np.abs(xhat) * mean_of(np.abs(dz * g * xhat))
    off = off_dz * np.abs(g)
    off_hat = np.abs(dz * g) * off_x
    allowed = 1.2 * r * (300 * ULP * terms + off + mean_of(off) + np.abs(xhat) * mean_of(off * np.abs(xhat) + off_hat) + off_x * mean_of(np.abs(dz * g * xhat)))
    assert (np.abs(c.maps(dx.host()) - want) <= allowed + half * (np.abs(want) + allowed)).all()
    assert dx.untouched_around()
    chain = (300 + c.images / 64) * ULP
    total = lambda a: np.abs(a).sum(axis=(0, 1))  # noqa: E731
    assert (np.abs(db.double().cpu().numpy() - want_b) <= chain * total(dz) + total(off_dz)).all()
    assert (np.abs(dg.double().cpu().numpy() - want_g) <= 1.2 * (chain * total(dz * xhat) + total(off_dz * xhat) + total(dz * off_x))).all()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(precision, dtype, shape):
    if shape[1] * shape[2] // shape[3] > 1:
        check_backward(Case(*shape, dtype, act="none"), from_bytes=True, d_residual=False)
    check_backward(Case(*shape, dtype, act="relu", residual=True))


# groups of many channels, in pieces of 8 that hold one, two, four or eight segments of them; narrow slabs; more images than workgroups
WIDE = [(4, 165, 317, 1), (3, 96, 496, 4), (2, 200, 124, 1), (3, 46, 354, 3), (3, 756, 384, 32), (2, 1218, 16, 16), (1, 30, 4096, 1), (1, 900, 4000, 2), (300, 3, 34, 17),
        (600, 50, 12, 6), (2, 60, 6, 3)]


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("shape", WIDE)
@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_wide_groups_both_ways(precision, dtype, shape, act):
    check_forward(Case(*shape, dtype, act=act, residual=True, seed=6), kept=True)
    for from_bytes in (False, True):
        check_backward(Case(*shape, dtype, act=act, residual=from_bytes, seed=7), from_bytes, d_residual=from_bytes)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("place", [dict(), dict(room=1), dict(room=5, shift=3), dict(room=8, shift=8)])
@pytest.mark.parametrize("from_bytes", [False, True])
def test_backward_activations_of_strided_maps(precision, dtype, act, place, from_bytes):
    for shape in ((3, 50, 24, 4), (1, 6000, 24, 6)):
        check_backward(Case(*shape, dtype, act=act, residual=True, seed=1, **place), from_bytes)
        check_backward(Case(*shape, dtype, act=act, seed=1, **place), from_bytes, d_residual=False)


@pytest.mark.parametrize("which", ["dx", "d_residual"])
def test_backward_in_place_of_dy(which):
    for shape in ((2, 50, 32, 4), (1, 9000, 40, 8)):
        c = Case(*shape, torch.bfloat16, act="silu", residual=True)
        _, stats = c.forward()
        ws, size = c.workspace()

        def run(dx, dres):
            dg, db = torch.empty(c.channels, device=DEV), torch.empty(c.channels, device=DEV)
            P.ppll_group_norm_backward(c.cfg, rows(c.x), None, stats, c.g, c.b, rows(c.res), None, rows(c.dy), rows(dx), rows(dres), dg, db, ws, size, stream())
            return dx.view.clone(), dres.view.clone(), dg, db

        apart = run(c.empty(), c.empty())
        together = run(c.dy if which == "dx" else c.empty(), c.dy if which == "d_residual" else c.empty())
        assert all(torch.equal(a, b) for a, b in zip(apart, together))


def test_no_images():
    cfg = P.group_norm_config(P.FP32, 0, 5, 8, 2)
    assert P.ppll_group_norm_workspace_bytes(cfg) == 0
    dg, db = torch.full((8,), 7.0, device=DEV), torch.full((8,), 7.0, device=DEV)
    P.ppll_group_norm_forward(cfg, None, None, None, None, None, None, None, None, 0, stream())
    P.ppll_group_norm_backward(cfg, None, None, None, None, None, None, None, None, None, None, dg, db, None, 0, stream())
    assert not dg.any() and not db.any()


def test_gradients_by_differences():
    c = Case(2, 6, 8, 2, torch.float32, act="silu", residual=True)
    y, stats = c.forward()
    dx, dres = c.empty(), c.empty()
    dg, db = torch.empty(8, device=DEV), torch.empty(8, device=DEV)
    ws, size = c.workspace()
    P.ppll_group_norm_backward(c.cfg, rows(c.x), None, stats, c.g, c.b, rows(c.res), None, rows(c.dy), rows(dx), rows(dres), dg, db, ws, size, stream())
    loss = lambda: float((c.forward()[0].host() * c.dy.host()).sum())  # noqa: E731
    h = 2.0 ** -6
    for t, grad in ((c.x.view, dx.view), (c.res.view, dres.view), (c.g.view(1, 8), dg.view(1, 8)), (c.b.view(1, 8), db.view(1, 8))):
        for i, j in ((0, 0), (t.shape[0] - 1, 5)):
            keep = float(t[i, j])
            t[i, j] = keep + h
            up = loss()
            t[i, j] = keep - h
            down = loss()
            t[i, j] = keep
            # third derivatives of order one: h^2 = 2.4e-4 of the largest slopes, and fp32 noise of the loss (1e-7) over h
            assert abs((up - down) / (2 * h) - float(grad[i, j])) <= 3 * h * h * float(grad.abs().max()) + 1e-4 * float(c.dy.view.abs().max())


@pytest.mark.parametrize("shape", [(6, 100, 32, 4), (2, 9000, 32, 4)])
def test_a_norm_as_it_is_used_captured_and_replayed(shape):
    """Forward that keeps its input in 8 bits, backward from those, in one graph on a stream of its own, replayed on new values."""
    c = Case(*shape, torch.bfloat16, act="relu", residual=True)
    side = torch.cuda.Stream()
    n = c.images * c.pixels
    keep = PlacedBytes(n, c.channels)
    y, dx, dres = c.empty(), c.empty(), c.empty()
    stats, dg, db = torch.empty(c.images, c.groups, 2, device=DEV), torch.empty(c.channels, device=DEV), torch.empty(c.channels, device=DEV)
    ws, size = c.workspace()

    def run():
        s = stream()
        P.ppll_group_norm_forward(c.cfg, rows(c.x), c.g, c.b, rows(c.res), rows(y), stats, P.byte_rows(keep.store, keep.exps), ws, size, s)
        P.ppll_group_norm_backward(c.cfg, None, P.byte_rows(keep.store, keep.exps), stats, c.g, c.b, None, rows(y), rows(c.dy), rows(dx), rows(dres), dg, db,
                                   ws, size, s)

    out = [y.view, dx.view, dres.view, stats, dg, db]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for seed in (1, 2, 3):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        for t in (c.x.view, c.res.view, c.dy.view):
            t.copy_(torch.randn(t.shape, generator=gen, device=DEV))
        run()
        torch.cuda.synchronize()
        eager = [t.clone() for t in out]
        for t in out:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, out))
    want, _, _ = c.oracle()
    assert np.abs(c.maps(y.host()) - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-3


def test_a_map_beyond_32_bits():
    # rows 49152 elements apart: the last ones lie beyond 2^31 elements
    n, ch, ld = 45000, 16, 49152
    store = torch.zeros(n * ld, dtype=torch.bfloat16, device=DEV).view(n, ld)
    x = store[:, -ch:]
    x.copy_(torch.randn(n, ch, device=DEV))
    y = store[:, :ch]
    g, b = torch.ones(ch, device=DEV), torch.zeros(ch, device=DEV)
    cfg = P.group_norm_config(P.BF16, 5, n // 5, ch, 2)
    ws = torch.empty(max(P.ppll_group_norm_workspace_bytes(cfg), 16), dtype=torch.uint8, device=DEV)
    P.ppll_group_norm_forward(cfg, P.rows(x), g, b, None, P.rows(y), None, None, ws, ws.numel(), stream())
    want, _, _ = O.group_norm_fwd(x.double().cpu().numpy().reshape(5, -1, ch), np.ones(ch), np.zeros(ch), 2, EPS)
    got = y.double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-5).all()
