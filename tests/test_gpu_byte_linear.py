"""The linear layer on rows of 8 bits, forward and backward, against 64-bit products of what the rows stand for.

Tolerances.  Forward: the whole-number sum is exact, its conversion, bias and residual are a rounding each of fp32, GELU's normal CDF is within 1e-6
(the rational approximation of erf within 1.5e-7, its exponential and reciprocal within a few 2^-22), the result a rounding of its type.  Backward:
products of a bf16 (or its three terms) and a value of 7 bits are exact in fp32, sums of K of them are off by 2^-23 of the sum of magnitudes for each addition at most."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from rows_helper import DEV, HALF, Placed, PlacedBytes, stream

pytestmark = pytest.mark.gpu
TYPES = [(P.FP32, torch.float32), (P.BF16, torch.bfloat16)]
ULP = 2.0 ** -24


class Layer:
    def __init__(self, rows, n_in, n_out, dtype, seed=0, room=0, shift=0, byte_room=0):
        rng = np.random.default_rng([seed, rows, n_in, n_out])
        self.rng, self.dtype, self.shape, self.place = rng, dtype, (rows, n_in, n_out), dict(room=room, shift=shift)
        self.qx, self.ex = rng.integers(-127, 128, (rows, n_in)), rng.integers(-9, -3, rows)
        self.qw, self.ew = rng.integers(-127, 128, (n_out, n_in)), rng.integers(-12, -8, n_out)
        self.x, self.w = PlacedBytes(rows, n_in, self.qx, self.ex, byte_room), PlacedBytes(n_out, n_in, self.qw, self.ew, byte_room)
        self.bias = torch.from_numpy(rng.standard_normal(n_out).astype(np.float32)).to(DEV)

    def cfg(self, act=P.ACT_NONE):
        return P.byte_linear_config(P.BF16 if self.dtype == torch.bfloat16 else P.FP32, *self.shape, act)

    def bytes(self, b):
        return P.byte_rows(b.store, b.exps)

    def values(self):
        return O.byte_values(self.qx, self.ex), O.byte_values(self.qw, self.ew)

    def put(self, *shape, scale=1.0):
        return Placed(scale * torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32)), self.dtype, **self.place)

    def empty(self, *shape):
        return Placed(shape, self.dtype, **self.place)


def rows(p):
    return None if p is None else P.rows(p.view)


def forward(l, gelu=False, residual=None, bias=True, slope=True):
    m, _, n = l.shape
    y, s = l.empty(m, n), l.empty(m, n) if gelu and slope else None
    P.ppll_byte_linear_forward(l.cfg(P.ACT_GELU if gelu else P.ACT_NONE), l.bytes(l.x), l.bytes(l.w), l.bias if bias else None, rows(residual), rows(y),
                               rows(s), stream())
    return y, s


def forward_on(kernel, l, gelu, residual):
    m, k, n = l.shape
    y, s = l.empty(m, n), l.empty(m, n) if gelu else None
    ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
    status = P.lib().ppll_internal_byte_linear(kernel, P.BF16 if l.dtype == torch.bfloat16 else P.FP32, m, k, n, int(gelu), ref(l.bytes(l.x)),
                                               ref(l.bytes(l.w)), ctypes.c_void_p(l.bias.data_ptr()), ref(rows(residual)), ref(rows(y)), ref(rows(s)),
                                               ctypes.c_void_p(stream()))
    assert status == 0, P.ppll_last_error()
    return y, s


def check_forward(l, gelu=False, with_residual=False, bias=True, kernel=None):
    m, _, n = l.shape
    residual = l.put(m, n) if with_residual else None
    y, s = forward(l, gelu, residual, bias) if kernel is None else forward_on(kernel, l, gelu, residual)
    x, w = l.values()
    h = x @ w.T
    size = np.abs(h)
    if bias:
        h = h + l.bias.double().cpu().numpy()
    if with_residual:
        h = h + residual.host()
        size = size + np.abs(residual.host())
    off = 3 * ULP * (size + np.abs(h) + 5)
    half = HALF[l.dtype]
    want = O.gelu_fwd(h) if gelu else h
    allowed = 1.2 * off + (1e-6 * np.abs(h) + 4 * ULP * np.abs(h) if gelu else 0)
    assert (np.abs(y.host() - want) <= allowed + half * (np.abs(want) + allowed)).all()
    assert y.untouched_around()
    if gelu:
        want = O.gelu_bwd(np.ones_like(h), h)
        allowed = off + 3e-6
        assert (np.abs(s.host() - want) <= allowed + half * (np.abs(want) + allowed)).all()
        assert s.untouched_around()


SIZES = [(1, 1, 1), (1, 16, 8), (1, 384, 1536), (2, 17, 9), (15, 64, 33), (16, 100, 100), (17, 130, 64), (33, 1000, 40), (64, 64, 64), (65, 128, 128),
         (66, 16, 200), (128, 65, 136), (129, 257, 127), (200, 48, 1000), (500, 333, 517), (1040, 384, 384)]


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("gelu,residual", [(False, False), (True, True)])
def test_forward(precision, dtype, size, gelu, residual):
    check_forward(Layer(*size, dtype), gelu, residual)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 40, 24), (70, 100, 90), (300, 64, 72)])
@pytest.mark.parametrize("place", [dict(room=1), dict(room=7, shift=3), dict(room=8, shift=8, byte_room=48)])
def test_forward_of_strided_rows(precision, dtype, size, place):
    check_forward(Layer(*size, dtype, seed=1, **place), True, True)
    check_forward(Layer(*size, dtype, seed=1, **place), False, False, bias=False)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("kernel", [1, 3, 4, 8, 10])
@pytest.mark.parametrize("size,place", [((1, 16, 8), {}), ((130, 1, 9), dict(room=3)), ((321, 33, 264), {}), ((700, 200, 520), dict(room=8, shift=8)),
                                        ((257, 513, 255), dict(room=1, shift=1)), ((640, 1000, 256), {})])
def test_each_kernel(precision, dtype, kernel, size, place):
    check_forward(Layer(*size, dtype, seed=2, **place), True, True, kernel=kernel)
    check_forward(Layer(*size, dtype, seed=2, **place), kernel=kernel)


@pytest.mark.parametrize("size", [(8320, 384, 1536), (20000, 200, 1536), (9000, 256, 264), (30000, 64, 768), (33000, 130, 512), (50000, 32, 256), (100001, 40, 20), (3000, 100, 33), (40, 300, 6100)])
def test_forward_of_many_rows(size):
    # every kind of tile that the rules choose among
    m, k, n = size
    l = Layer(300, k, n, torch.bfloat16)
    times = -(-m // 300)
    x, e = l.x.store.repeat(times, 1)[:m].contiguous(), l.x.exps[:300].repeat(times)[:m].contiguous()
    y, out = torch.empty(m, n, dtype=torch.bfloat16, device=DEV), torch.empty(300, n, dtype=torch.bfloat16, device=DEV)
    P.ppll_byte_linear_forward(l.cfg(), l.bytes(l.x), l.bytes(l.w), l.bias, None, P.rows(out), None, stream())
    P.ppll_byte_linear_forward(P.byte_linear_config(P.BF16, m, k, n), P.byte_rows(x, e), l.bytes(l.w), l.bias, None, P.rows(y), None, stream())
    assert torch.equal(y, out.repeat(times, 1)[:m])
    check_forward(l)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows_", [3, 100])
def test_forward_of_extreme_exponents_and_rows_of_nan(precision, dtype, rows_):
    l = Layer(rows_, 48, 20, dtype)
    l.x.exps[0], l.x.exps[1], l.w.exps[4], l.w.exps[5] = -128, 121, -128, -126
    l.x.store[2] = 0
    y, _ = forward(l)
    y = y.host()
    assert np.isnan(y[0]).all() and np.isnan(y[:, 4]).all()
    keep = np.ones(20, dtype=bool)
    keep[4] = False
    assert np.array_equal(y[2, keep], l.bias.cpu().to(dtype).double().numpy()[keep])     # zeros times any step
    l.ex[0], l.ex[1], l.ew[4], l.ew[5] = 0, 121, 0, -126
    x, w = l.values()
    with np.errstate(over="ignore"):
        want = torch.from_numpy((x[1] @ w.T) + l.bias.double().cpu().numpy()).to(torch.float32).to(dtype).double().numpy()
    fine = np.isfinite(want) & keep
    assert np.array_equal(np.isinf(y[1])[keep], np.isinf(want)[keep])
    assert (np.abs(y[1] - want)[fine] <= 3 * HALF[dtype] * np.abs(want)[fine] + 1e-6).all()


def test_forward_of_the_largest_sums():
    # 65536 products of 127 x 127, and with a caller's own -128
    l = Layer(2, 65536, 3, torch.float32)
    l.x.store[:], l.w.store[:] = 127, 127
    l.x.exps[:], l.w.exps[:] = 0, 0
    l.w.store[1], l.w.store[2] = -127, -128
    l.x.store[1] = -128
    y, _ = forward(l, bias=False)
    want = 65536.0 * np.array([[127 * 127, -127 * 127, -127 * 128], [-128 * 127, 128 * 127, 128 * 128]])
    assert np.array_equal(y.host(), want)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows_", [3, 100, 400])
def test_forward_of_steps_below_the_types_range(precision, dtype, rows_):
    """A step of 2^-160 is none in fp32, 2^26 of them are a number (a subnormal one)."""
    l = Layer(rows_, 4096, 20, dtype)
    l.x.exps[:rows_], l.w.exps[:20] = -100, -60
    l.x.exps[1] = -90
    l.x.store[:], l.w.store[:] = 127, 127
    l.w.store[3] = -127
    y, _ = forward(l, bias=False)
    want = np.full((rows_, 20), 4096 * 127 * 127 * 2.0 ** -160)
    want[1] *= 2.0 ** 10
    want[:, 3] *= -1
    smallest = 2.0 ** (-149 if dtype == torch.float32 else -133)
    assert (np.abs(y.host() - want) <= HALF[dtype] * np.abs(want) + smallest / 2).all()
    assert (y.host()[1] != 0).all()


def test_forward_in_place_of_the_residual():
    l = Layer(70, 64, 48, torch.bfloat16)
    residual = l.put(70, 48)
    y, _ = forward(l, residual=residual)
    P.ppll_byte_linear_forward(l.cfg(), l.bytes(l.x), l.bytes(l.w), l.bias, rows(residual), rows(residual), None, stream())
    assert torch.equal(residual.view, y.view)


def check_backward(l, gate=False, want=("dx", "dw", "db"), seed_scale=1e-3, way=None):
    m, k, n = l.shape
    dy, g = l.put(m, n, scale=seed_scale), l.put(m, k) if gate else None
    dx = l.empty(m, k) if "dx" in want else None
    dw = torch.full((k, n), 7.0, device=DEV) if "dw" in want else None
    db = torch.full((n,), 7.0, device=DEV) if "db" in want else None
    if way is None:
        size = P.ppll_byte_linear_workspace_bytes(l.cfg())
        ws = torch.full((max(size, 16) + 64,), 0x77, dtype=torch.uint8, device=DEV)
        P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), rows(g), rows(dx), dw, db, ws, size, stream())
    else:
        n_bytes = ctypes.c_size_t(0)
        ref = lambda r: None if r is None else ctypes.byref(r)  # noqa: E731
        ptr = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())  # noqa: E731
        call = lambda ws_: P.lib().ppll_internal_byte_linear_backward(way, m, k, n, ref(l.bytes(l.x)), ref(l.bytes(l.w)), ref(rows(dy)), ref(rows(g)),  # noqa: E731
                                                                      ref(rows(dx)), ptr(dw), ptr(db), ws_, ctypes.byref(n_bytes), ctypes.c_void_p(stream()))
        assert call(None) == 0
        size = n_bytes.value
        ws = torch.full((max(size, 16) + 64,), 0x77, dtype=torch.uint8, device=DEV)
        assert call(ptr(ws)) == 0, P.ppll_last_error()
    x, w = l.values()
    d, half = dy.host(), HALF[l.dtype]
    if dx is not None:
        ref, size_of = d @ w, np.abs(d) @ np.abs(w)
        allowed = (n + 2) * 2 * ULP * size_of
        if gate:
            ref, allowed = ref * g.host(), (allowed + ULP * np.abs(ref)) * np.abs(g.host())
        assert (np.abs(dx.host() - ref) <= allowed + half * (np.abs(ref) + allowed)).all()
        assert dx.untouched_around()
    if dw is not None:
        ref = x.T @ d
        assert (np.abs(dw.double().cpu().numpy() - ref) <= (m + 2) * 2 * ULP * (np.abs(x).T @ np.abs(d))).all()
    if db is not None:
        assert (np.abs(db.double().cpu().numpy() - d.sum(0)) <= (m + 2) * ULP * np.abs(d).sum(0)).all()
    assert bool((ws[size:] == 0x77).all())
    return dx, dw, db


BACK = [(1, 1, 1), (1, 16, 8), (2, 5, 3), (3, 7, 200), (8, 200, 7), (16, 64, 64), (31, 40, 17), (64, 128, 128), (65, 129, 130), (127, 33, 257), (128, 24, 40),
        (300, 201, 333), (777, 100, 61), (1000, 256, 8)]


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", BACK)
@pytest.mark.parametrize("gate", [False, True])
def test_backward(precision, dtype, size, gate):
    check_backward(Layer(*size, dtype), gate)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", [(40, 24, 16), (200, 130, 90)])
@pytest.mark.parametrize("place", [dict(room=1), dict(room=7, shift=3), dict(room=8, shift=8, byte_room=48)])
def test_backward_of_strided_rows(precision, dtype, size, place):
    check_backward(Layer(*size, dtype, seed=1, **place), True)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("db",), ("dw", "db"), ("dx", "db")])
def test_gradients_that_are_not_wanted(precision, dtype, want):
    for rows_ in (5, 700, 2000):
        check_backward(Layer(rows_, 72, 40, dtype), False, want)


@pytest.mark.parametrize("way", [1, 2])
@pytest.mark.parametrize("size", [(1, 16, 8), (70, 40, 24), (333, 136, 200), (1000, 520, 264), (2500, 24, 72)])
@pytest.mark.parametrize("want", [("dx", "dw", "db"), ("dx",), ("dw",)])
def test_each_way_backward(way, size, want):
    check_backward(Layer(*size, torch.bfloat16, seed=3, room=8), "dx" in want, want, way=way)


def test_backward_of_a_wide_layer():
    # as values by the rules, both gradients and dX alone
    l = Layer(4100, 1536, 3200, torch.bfloat16)
    m, k, n = l.shape
    x, w = (torch.from_numpy(v).to(DEV).float() for v in l.values())
    dy = l.put(m, n)
    d = dy.view.float()
    dx, dw, db = l.empty(m, k), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
    size = P.ppll_byte_linear_workspace_bytes(l.cfg())
    ws = torch.full((size + 64,), 0x77, dtype=torch.uint8, device=DEV)
    P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx), dw, db, ws, size, stream())
    both = dx.view.clone()
    # against fp32 products, each side off by the roundings of its sums
    for got, want, count in ((both.float(), d @ w, n), (dw, x.t().contiguous() @ d, m)):
        size_of = (d.abs() @ w.abs()) if count == n else (x.abs().t().contiguous() @ d.abs())
        assert bool(((got - want).abs() <= 4 * count * ULP * size_of + (2 ** -8 * want.abs() if count == n else 0)).all())
    assert bool(((db.double() - d.double().sum(0)).abs() <= m * ULP * d.double().abs().sum(0)).all())
    P.ppll_byte_linear_backward(l.cfg(), None, l.bytes(l.w), rows(dy), None, rows(dx), None, None, ws, size, stream())
    assert torch.equal(dx.view, both) and bool((ws[size:] == 0x77).all())


@pytest.mark.parametrize("size", [(1, 16, 4096), (20, 88, 1344), (60, 224, 2432), (128, 1024, 4096), (499, 1632, 3352), (640, 768, 2304)])
def test_backward_of_few_rows_and_many_channels(size):
    # as values by the rules; with rows that do not lie whole the same gradients on the other way
    check_backward(Layer(*size, torch.bfloat16, seed=5), True)
    check_backward(Layer(*size, torch.bfloat16, seed=5, room=1), True)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size", [(1, 1, 2000), (5, 203, 1111), (41, 63, 1645), (130, 19, 777), (129, 300, 1030), (260, 131, 2051), (2, 8, 65536)])
@pytest.mark.parametrize("want", [("dx", "dw", "db"), ("dx",), ("dx", "db")])
def test_dx_in_parts_of_its_channels(precision, dtype, size, want):
    check_backward(Layer(*size, dtype, seed=8, room=3), True, want)


def test_backward_of_many_rows():
    check_backward(Layer(8320, 384, 128, torch.bfloat16), True)
    check_backward(Layer(20000, 40, 24, torch.bfloat16))
    check_backward(Layer(9000, 24, 40, torch.float32))


def test_column_sums_of_more_rows_than_a_grid_has_stretches_of():
    m = (1 << 24) + 700
    for dtype, precision in ((torch.bfloat16, P.BF16), (torch.float32, P.FP32)):
        dy = torch.randint(-1, 2, (m, 2), device=DEV).to(dtype)      # whole sums, exact in fp32
        cfg, db = P.byte_linear_config(precision, m, 1, 2), torch.empty(2, device=DEV)
        ws = torch.empty(P.ppll_byte_linear_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
        P.ppll_byte_linear_backward(cfg, None, None, P.rows(dy), None, None, None, db, ws, ws.numel(), stream())
        assert torch.equal(db.double(), dy.double().sum(0))


def test_backward_of_rows_far_apart():
    # 2^20 elements between rows of dy, dx and gate in turn: more than 32 bits of bytes over all of them
    m, k, n = 1100, 64, 64
    l = Layer(m, k, n, torch.bfloat16)
    near = {name: torch.randn(m, 64, device=DEV).bfloat16() for name in ("dy", "gate", "dx")}
    store = torch.zeros(m << 20, dtype=torch.bfloat16, device=DEV).view(m, 1 << 20)
    ws = torch.empty(P.ppll_byte_linear_workspace_bytes(l.cfg()), dtype=torch.uint8, device=DEV)

    def run(dw, **other):
        t = {**near, **other}
        P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), P.rows(t["dy"]), P.rows(t["gate"]), P.rows(t["dx"]), dw, None, ws, ws.numel(), stream())
        return t["dx"].double().cpu()
    x, w = l.values()
    d, g = near["dy"].double().cpu().numpy(), near["gate"].double().cpu().numpy()
    want = (d @ w) * g
    allowed = ((n + 2) * 2 * ULP * (np.abs(d) @ np.abs(w)) + ULP * np.abs(d @ w)) * np.abs(g)
    for name in ("dy", "gate", "dx"):
        far = store[:, -64:]
        far.copy_(near[name])
        for dw in (None, torch.empty(k, n, device=DEV)):
            got = run(dw, **{name: far}).numpy()
            assert (np.abs(got - want) <= allowed + HALF[torch.bfloat16] * (np.abs(want) + allowed)).all()
            if dw is not None:
                assert (np.abs(dw.double().cpu().numpy() - x.T @ d) <= (m + 2) * 2 * ULP * (np.abs(x).T @ np.abs(d))).all()
        store.zero_()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("size,dw", [((300, 70, 40), True), ((700, 128, 64), False), ((700, 128, 64), True), ((8192, 1536, 1536), True)])
def test_dx_in_place_of_the_gate(precision, dtype, size, dw):
    m, k, n = size
    l = Layer(*size, dtype)
    dy, gate, dx = l.put(m, n), l.put(m, k), l.empty(m, k)
    ws = torch.empty(max(P.ppll_byte_linear_workspace_bytes(l.cfg()), 16), dtype=torch.uint8, device=DEV)
    go = lambda to: P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), rows(gate), rows(to),  # noqa: E731
                                                torch.empty(k, n, device=DEV) if dw else None, None, ws, ws.numel(), stream())
    go(dx)
    go(gate)
    assert torch.equal(dx.view, gate.view)


def test_the_sums_have_a_fixed_order_and_need_nothing_of_the_workspace():
    for m, k, n in ((3000, 130, 70), (90, 72, 1500), (1000, 64, 1100)):
        l = Layer(m, k, n, torch.bfloat16)
        dy = l.put(m, n)
        got = []
        size = P.ppll_byte_linear_workspace_bytes(l.cfg())
        for fill in (0, 0xff, 0x3c):
            dx, dw, db = l.empty(m, k), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
            ws = torch.full((size,), fill, dtype=torch.uint8, device=DEV)
            P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx), dw, db, ws, size, stream())
            got.append((dx.view, dw, db))
        for other in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_calls_on_two_streams_at_once():
    """Layers and norms with workspaces of their own, in flight together; results as one behind the other."""
    def make(seed):
        l = Layer(2500, 200, 600, torch.bfloat16, seed=seed)
        dy, n = l.put(2500, 600), P.ppll_byte_linear_workspace_bytes(l.cfg())
        norm = P.group_norm_config(P.BF16, 25, 100, 200, 8, P.ACT_SILU, 1e-5)
        k = P.ppll_group_norm_workspace_bytes(norm)
        scale = torch.linspace(0.5, 2, 200, device=DEV)

        def go():
            ws, ws2 = (torch.empty(max(b, 16), dtype=torch.uint8, device=DEV) for b in (n, k))
            y, dx, dw, db = l.empty(2500, 600), l.empty(2500, 200), torch.empty(200, 600, device=DEV), torch.empty(600, device=DEV)
            dn, stats, dg, dh = l.empty(2500, 200), torch.empty(25, 8, 2, device=DEV), torch.empty(200, device=DEV), torch.empty(200, device=DEV)
            s = torch.cuda.current_stream().cuda_stream
            for _ in range(5):
                P.ppll_byte_linear_forward(l.cfg(), l.bytes(l.x), l.bytes(l.w), l.bias, None, rows(y), None, s)
                P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx), dw, db, ws, n, s)
                P.ppll_group_norm_forward(norm, rows(dx), scale, scale, None, rows(dn), stats, None, ws2, k, s)
                P.ppll_group_norm_backward(norm, rows(dx), None, stats, scale, scale, None, None, rows(dn), rows(dn), None, dg, dh, ws2, k, s)
            return [y.view, dx.view, dw, db, dn.view, stats, dg, dh], (ws, ws2)
        return go
    calls = [make(seed) for seed in (1, 2)]
    want = [go()[0] for go in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in calls], []
    for _ in range(3):
        for go, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(go())
    torch.cuda.synchronize()
    for i, (g, _) in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2]))


def test_no_rows():
    l = Layer(1, 24, 16, torch.bfloat16)
    cfg = P.byte_linear_config(P.BF16, 0, 24, 16)
    dw, db = torch.full((24, 16), 7.0, device=DEV), torch.full((16,), 7.0, device=DEV)
    P.ppll_byte_linear_forward(cfg, None, None, None, None, None, None, stream())
    P.ppll_byte_linear_backward(cfg, None, None, None, None, None, dw, db, None, 0, stream())
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("precision,dtype", TYPES)
def test_rows_of_nan_reach_what_they_are_part_of(precision, dtype):
    l = Layer(70, 40, 24, dtype)
    l.x.exps[3], l.w.exps[5] = -128, -128
    l.x.store[3], l.w.store[5] = 0, 0
    dy = l.put(70, 24)
    dx, dw, db = l.empty(70, 40), torch.empty(40, 24, device=DEV), torch.empty(24, device=DEV)
    size = P.ppll_byte_linear_workspace_bytes(l.cfg())
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)
    P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx), dw, db, ws, size, stream())
    assert np.isnan(dx.host()).all() and bool(dw.isnan().all()) and bool(db.isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_by_differences(dtype):
    # y is linear in the weight's and the tokens' values: a change of one q by one is a change of y by the other side's value
    l = Layer(6, 20, 9, torch.float32)
    m, k, n = l.shape
    dy = Placed(torch.from_numpy(l.rng.standard_normal((m, n)).astype(np.float32)).to(dtype).float(), torch.float32)
    dx, dw, db = l.empty(m, k), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV)
    P.ppll_byte_linear_backward(l.cfg(), l.bytes(l.x), l.bytes(l.w), rows(dy), None, rows(dx), dw, db, torch.empty(16, dtype=torch.uint8, device=DEV),
                                P.ppll_byte_linear_workspace_bytes(l.cfg()), stream())
    loss = lambda: float((forward(l)[0].host() * dy.host()).sum())  # noqa: E731
    for store, exps, grad in ((l.x.store, l.ex, lambda i, j: dx.host()[i, j]), (l.w.store, l.ew, lambda i, j: float(dw[j, i]))):
        for i, j in ((0, 0), (3, 7), (5, 19)):
            keep = int(store[i, j])
            store[i, j] = min(keep + 1, 127)
            up, high = loss(), min(keep + 1, 127)
            store[i, j] = max(keep - 1, -127)
            down, low = loss(), max(keep - 1, -127)
            store[i, j] = keep
            # y is off by 3 roundings of its size (some 60) each way, weighted by dy
            room = 2 * 6 * ULP * 60 * np.abs(dy.host()).sum()
            assert abs((up - down) - (high - low) * 2.0 ** exps[i] * grad(i, j)) <= room


def test_a_layer_as_it_is_used_captured_and_replayed():
    """Tokens and weight into 8 bits, forward, backward, in one graph on a stream of its own, replayed on new values."""
    m, k, n = 300, 96, 72
    side = torch.cuda.Stream()
    x, w, bias, dy = torch.empty(m, k, device=DEV, dtype=torch.bfloat16), torch.empty(k, n, device=DEV), torch.empty(n, device=DEV), torch.empty(m, n, device=DEV, dtype=torch.bfloat16)
    new8 = lambda r, c: (torch.empty(r, (c + 15) // 16 * 16, dtype=torch.int8, device=DEV), torch.empty(r, dtype=torch.int8, device=DEV))  # noqa: E731
    x8, w8 = new8(m, k), new8(n, k)
    cfg = P.byte_linear_config(P.BF16, m, k, n, P.ACT_GELU)
    out = {"y": torch.empty(m, n, device=DEV, dtype=torch.bfloat16), "slope": torch.empty(m, n, device=DEV, dtype=torch.bfloat16),
           "dx": torch.empty(m, k, device=DEV, dtype=torch.bfloat16), "dw": torch.empty(k, n, device=DEV), "db": torch.empty(n, device=DEV)}
    ws = torch.empty(max(P.ppll_byte_linear_workspace_bytes(cfg), 16), dtype=torch.uint8, device=DEV)

    def run():
        s = stream()
        P.ppll_byte_rows_pack(P.BF16, m, k, P.rows(x), P.byte_rows(*x8), s)
        P.ppll_byte_rows_pack_columns(P.FP32, k, n, P.rows(w), P.byte_rows(*w8), s)
        P.ppll_byte_linear_forward(cfg, P.byte_rows(*x8), P.byte_rows(*w8), bias, None, P.rows(out["y"]), P.rows(out["slope"]), s)
        P.ppll_byte_linear_backward(cfg, P.byte_rows(*x8), P.byte_rows(*w8), P.rows(dy), None, P.rows(out["dx"]), out["dw"], out["db"], ws, ws.numel(), s)

    def fill(seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        for t in (x, w, bias, dy):
            t.copy_(torch.randn(t.shape, generator=gen, device=DEV))

    with torch.cuda.stream(side):
        fill(0)
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for seed in (1, 2, 3):
        fill(seed)
        run()
        torch.cuda.synchronize()
        eager = {k_: v.clone() for k_, v in out.items()}
        for v in out.values():
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eager[k_], out[k_]) for k_ in out)
    qx, ex = O.byte_rows(x.double().cpu().numpy())
    qw, ew = O.byte_rows(w.double().cpu().numpy().T)
    vx, vw = O.byte_values(qx, ex), O.byte_values(qw, ew)
    h = vx @ vw.T + bias.double().cpu().numpy()
    want = O.gelu_fwd(h)
    assert (np.abs(out["y"].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 4e-6 * (1 + np.abs(h))).all()
