"""Norm and rotary positions of queries and keys, forward and backward, against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # a rounding, relative


def stream():
    return torch.cuda.current_stream().cuda_stream


class Case:
    def __init__(self, batch=2, tokens=5, q_heads=2, k_heads=2, head_dim=16, pairs=(4, 4), base=100.0, neighbours=False, norm=True, eps=1e-6,
                 dtype=torch.float32, far=20, room=(0, 0), shift=0, seed=0):
        rng = np.random.default_rng([seed, tokens, head_dim, q_heads])
        self.__dict__.update({k: v for k, v in locals().items() if k not in ("self", "rng")})
        self.rows = batch * tokens
        self.positions = rng.integers(-far if far < 1 << 30 else -(1 << 31), far, (tokens, len(pairs))).astype(np.int32)
        self.cfg = P.rotary_config(P.BF16 if dtype == torch.bfloat16 else P.FP32, self.rows, tokens, q_heads, k_heads, head_dim, pairs, base,
                                   neighbours, eps)
        self.scales = [(1 + 0.3 * rng.standard_normal(head_dim)).astype(np.float32) if norm else None for _ in range(2)]
        self.x = [self.rows_of(rng, h) for h in (q_heads, k_heads)]
        self.dy = [self.rows_of(rng, h) for h in (q_heads, k_heads)]
        self.pos_dev = torch.from_numpy(self.positions).to(DEV)
        self.scale_dev = [None if s is None or not h else torch.from_numpy(s).to(DEV) for s, h in zip(self.scales, (q_heads, k_heads))]

    def rows_of(self, rng, heads):
        return torch.from_numpy(rng.standard_normal((self.rows, heads * self.head_dim)).astype(np.float32)).to(DEV, self.dtype)

    def place(self, values=None):
        """Rows with room on both sides of them (7 where nothing was put), `shift` elements off the allocation's alignment."""
        out = []
        for i, h in enumerate((self.q_heads, self.k_heads)):
            w = h * self.head_dim
            store = torch.full((self.rows * (w + self.room[i]) + self.shift + 16,), 7.0, dtype=self.dtype, device=DEV)
            v = store[self.shift:self.shift + self.rows * (w + self.room[i])].view(self.rows, w + self.room[i])[:, self.room[i] // 2:][:, :w]
            if values is not None:
                v.copy_(values[i])
            out.append((store, v))
        return out

    def sides(self, placed):
        v = [None if not h else p[1] for p, h in zip(placed, (self.q_heads, self.k_heads))]
        return P.QueriesKeys(*(None if t is None else t.data_ptr() for t in v), *(0 if t is None else self.room[i] + t.shape[1] for i, t in enumerate(v)))

    def rest_is(self, placed, value=7.0):
        for i, (store, v) in enumerate(placed):
            keep = v.clone()
            v.fill_(value)
            assert (store == value).all()
            v.copy_(keep)

    def heads(self, t):
        return t.double().cpu().numpy().reshape(self.batch, self.tokens, -1, self.head_dim)

    def angles(self):
        return O.rotary_angles(self.positions, self.pairs, np.float32(self.base))

    def want_forward(self, side):
        x = self.heads(self.x[side])
        if self.norm:
            x = O.rms_norm_fwd(x, self.scales[side].astype(np.float64), float(np.float32(self.eps)))[0]
        return O.rotate(x, self.angles(), self.neighbours)

    def want_backward(self, side):
        dz = O.rotate(self.heads(self.dy[side]), -self.angles(), self.neighbours)
        if not self.norm:
            return dz, None
        g = self.scales[side].astype(np.float64)
        return O.rms_norm_bwd(dz, O.rms_norm_fwd(self.heads(self.x[side]), g, float(np.float32(self.eps)))[1], g)

    def arithmetic(self):
        """fp32 roundings on the way to an element, beside the size of its head's largest: angle 2^-23 (turn of up to 1/2 kept to 2^-25, times
        2 pi), cos and sin 2 each, two products and a sum, and with the norm a sum over the head, a root, a quotient and two products more."""
        return (10 + (8 + self.head_dim ** 0.5 if self.norm else 0)) * 2.0 ** -24

    def forward(self, in_place=False, keep=False):
        x = self.place(self.x)
        y = x if in_place else self.place()
        kept = self.place() if keep else None
        P.ppll_qk_rotary_forward(self.cfg, self.pos_dev, *self.scale_dev, self.sides(x), self.sides(y), self.sides(kept) if keep else None, stream())
        torch.cuda.synchronize()
        for side, heads in enumerate((self.q_heads, self.k_heads)):
            if heads:
                self.close(y[side][1], self.want_forward(side), self.arithmetic())
                if keep:
                    assert torch.equal(kept[side][1], self.x[side])
                if not in_place:
                    assert torch.equal(x[side][1], self.x[side])
        self.rest_is(y)
        return y

    def close(self, got, want, eps, more=0.0):
        got = self.heads(got)
        size = np.abs(want).max(-1, keepdims=True)
        limit = HALF[self.dtype] * np.abs(want) * 1.01 + eps * size * 4 + more + 1e-30
        worst = (np.abs(got - want) / limit).max()      # NaN if anything is
        assert worst <= 1

    def backward(self, in_place=False):
        x, dy = self.place(self.x), self.place(self.dy)
        dx = dy if in_place else self.place()
        ds = [torch.full((self.head_dim + 3,), 9.0, device=DEV) for _ in range(2)]
        n = P.ppll_qk_rotary_workspace_bytes(self.cfg) if self.norm else 0
        ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None
        have = lambda v: [t if h and self.norm else None for t, h in zip(v, (self.q_heads, self.k_heads))]  # noqa: E731
        P.ppll_qk_rotary_backward(self.cfg, self.pos_dev, *self.scale_dev, self.sides(x) if self.norm else None, self.sides(dy), self.sides(dx),
                                  *have(ds), ws, n, stream())
        torch.cuda.synchronize()
        for side, heads in enumerate((self.q_heads, self.k_heads)):
            if not heads:
                continue
            want, dscale = self.want_backward(side)
            # the gradient's two terms cancel: roundings are of the size of dz r, the larger of them
            r = O.rms_norm_fwd(self.heads(self.x[side]), 1.0, float(np.float32(self.eps)))[1][1] if self.norm else 1.0
            size = np.abs(self.heads(self.dy[side])).max(-1, keepdims=True) * r * (np.abs(self.scales[side]).max() if self.norm else 1.0)
            self.close(dx[side][1], want, self.arithmetic(), 8 * self.arithmetic() * size)
            if self.norm:
                terms = self.rows * heads
                each = np.abs(self.heads(self.dy[side])).max() * self.head_dim ** 0.5       # |x r| is at most sqrt(head_dim)
                got = ds[side].double().cpu().numpy()
                assert (np.abs(got[:self.head_dim] - dscale) <= 4 * self.arithmetic() * each * terms ** 0.5 + 2 ** -24 * np.abs(dscale) * 8).all()
                assert (got[self.head_dim:] == 9).all()
        self.rest_is(dx)
        return dx, ds


DTYPES = [torch.float32, torch.bfloat16]
# head widths with whole 16-byte pieces of half a head, with 8-byte ones, with neither; heads that turn in part; one, two, three axes
HEADS = [(16, (4, 4)), (64, (16, 16)), (128, (16, 24, 24)), (128, (24, 20, 20)), (256, (128,)), (40, (10, 10)), (72, (12, 12, 12)), (96, (48,)), (80, (20, 20)),
         (6, (1, 1, 1)), (2, (1,)), (34, (17,)), (64, (8, 8)), (64, (5, 0, 3)), (48, (0, 24)), (24, (0,)), (250, (60, 65)), (256, (10,))]


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("head_dim,pairs", HEADS)
def test_heads(head_dim, pairs, dtype, norm, neighbours):
    c = Case(head_dim=head_dim, pairs=pairs, dtype=dtype, norm=norm, neighbours=neighbours, q_heads=3, k_heads=1, batch=3, tokens=7)
    c.forward()
    c.backward()


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("batch,tokens,q_heads,k_heads", [(1, 1, 1, 1), (1, 1, 1, 0), (3, 1, 0, 2), (1, 700, 4, 2), (33, 65, 6, 6), (1, 9001, 2, 1), (5, 13, 40, 8),
                                                          (2, 3, 130, 1)])
def test_rows_and_heads(batch, tokens, q_heads, k_heads, norm):
    c = Case(batch=batch, tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=64, pairs=(16, 16), dtype=torch.bfloat16, norm=norm)
    c.forward(keep=True)
    c.backward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("room,shift", [((0, 0), 0), ((64, 8), 0), ((16, 32), 8), ((3, 5), 0), ((0, 0), 1), ((8, 8), 4), ((4, 12), 2)])
def test_strides_and_alignment_and_in_place(room, shift, dtype):
    for norm in (False, True):
        c = Case(head_dim=32, pairs=(8, 8), q_heads=4, k_heads=2, batch=2, tokens=9, room=room, shift=shift, dtype=dtype, norm=norm)
        y, z = c.forward(), c.forward(in_place=True, keep=True)
        assert all(torch.equal(a[1], b[1]) for a, b in zip(y, z))
        (a, s), (b, t) = c.backward(), c.backward(in_place=True)
        assert all(torch.equal(u[1], v[1]) for u, v in zip(a, b)) and all(torch.equal(u, v) for u, v in zip(s, t))


@pytest.mark.parametrize("far,base", [(1 << 20, 10000.0), (1 << 31, 100.0), (1 << 31, 1.0), (100, 1e6), (50, 0.5)])
def test_far_positions(far, base):
    for neighbours in (False, True):
        c = Case(tokens=40, far=far, base=base, neighbours=neighbours, head_dim=64, pairs=(12, 10, 10), norm=False)
        c.forward()
        c.backward()


def test_zero_rows_and_small_values():
    # a head of zeros has no direction: eps alone is under the root
    c = Case(head_dim=64, pairs=(16, 16), tokens=6, q_heads=2, k_heads=2, eps=1e-2)
    for t in c.x:
        t[2].zero_()
        t[3] *= 1e-12
        t[4] *= 1e12
    y = c.forward()
    assert (y[0][1][2] == 0).all()
    c.backward()


def test_values_that_are_not_finite_stay_in_their_head():
    c = Case(head_dim=64, pairs=(16, 16), tokens=6, q_heads=2, k_heads=1)
    c.x[0][1, 5], c.x[0][4, 64] = float("nan"), float("inf")
    x, y = c.place(c.x), c.place()
    P.ppll_qk_rotary_forward(c.cfg, c.pos_dev, *c.scale_dev, c.sides(x), c.sides(y), None, stream())
    torch.cuda.synchronize()
    bad = ~torch.isfinite(y[0][1].view(-1, 2, 64)).all(-1)
    assert bad.nonzero().tolist() == [[1, 0], [4, 1]] and torch.isfinite(y[1][1]).all()


def test_no_rows_leave_gradients_of_zero():
    cfg = P.rotary_config(P.BF16, 0, 4, 2, 2, 64, [16, 16], 100.0)
    s = torch.ones(64, device=DEV)
    ds = [torch.full((64,), 5.0, device=DEV) for _ in range(2)]
    P.ppll_qk_rotary_backward(cfg, None, s, s, None, None, None, *ds, None, 0, stream())
    torch.cuda.synchronize()
    assert all((d == 0).all() for d in ds)


def test_gradients_against_differences():
    c = Case(batch=1, tokens=3, q_heads=2, k_heads=1, head_dim=10, pairs=(2, 2), norm=True, eps=0.1)
    dx, ds = c.backward()
    side, h = 0, 1e-5
    f = lambda: (c.want_forward(side) * c.heads(c.dy[side])).sum()  # noqa: E731
    x = c.x[side].double()
    want = np.zeros(x.shape)
    for r in range(x.shape[0]):
        for e in range(x.shape[1]):
            c.x[side] = x.clone()
            c.x[side][r, e] += h
            up = f()
            c.x[side][r, e] -= 2 * h
            want[r, e] = (up - f()) / (2 * h)
    c.x[side] = x
    # differences in 64 bits: h^2 and 1e-16 / h; the kernel in 32
    assert np.abs(dx[side][1].double().cpu().numpy() - want).max() <= 1e-5 * np.abs(want).max()
    g = c.scales[side].astype(np.float64)
    for e in range(10):
        c.scales[side] = g + h * (np.arange(10) == e)
        up = f()
        c.scales[side] = g - h * (np.arange(10) == e)
        assert abs(ds[side][e].item() - (up - f()) / (2 * h)) <= 1e-5 * max(1.0, abs(up))


@pytest.mark.parametrize("norm", [False, True])
def test_captured_and_replayed(norm):
    c = Case(head_dim=64, pairs=(16, 16), batch=4, tokens=65, q_heads=6, k_heads=6, dtype=torch.bfloat16, norm=norm)
    x, y, dy, dx = c.place(c.x), c.place(), c.place(c.dy), c.place()
    ds = [torch.empty(64, device=DEV) for _ in range(2)]
    n = P.ppll_qk_rotary_workspace_bytes(c.cfg)
    ws, other = (torch.full((n,), 255, dtype=torch.uint8, device=DEV) for _ in range(2))

    def both(y, dx, ds, ws):
        P.ppll_qk_rotary_forward(c.cfg, c.pos_dev, *c.scale_dev, c.sides(x), c.sides(y), None, stream())
        P.ppll_qk_rotary_backward(c.cfg, c.pos_dev, *c.scale_dev, c.sides(x) if norm else None, c.sides(dy), c.sides(dx), *(ds if norm else (None, None)),
                                  ws, n, stream())

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        both(y, dx, ds, ws)
    y2, dx2, ds2 = c.place(), c.place(), [torch.empty(64, device=DEV) for _ in range(2)]
    for k in range(3):
        for t in x + dy:
            t[1].mul_(-0.5 if k else 1.0)
        graph.replay()
        both(y2, dx2, ds2, other)
        torch.cuda.synchronize()
        assert all(torch.equal(a[1], b[1]) for a, b in zip(y + dx, y2 + dx2))
        assert not norm or all(torch.equal(a, b) for a, b in zip(ds, ds2))


def test_offsets_beyond_32_bits():
    # rows 2^26 elements apart: the last of 40 starts at element 2.6e9
    rows, ld = 40, 1 << 26
    store = torch.empty(rows * ld, dtype=torch.bfloat16, device=DEV)
    c = Case(batch=1, tokens=rows, q_heads=1, k_heads=0, head_dim=64, pairs=(16, 16), dtype=torch.bfloat16, norm=False)
    view = store.view(rows, ld)[:, :64]
    view.copy_(c.x[0])
    qk = P.QueriesKeys(view.data_ptr(), None, ld, 0)
    P.ppll_qk_rotary_forward(c.cfg, c.pos_dev, None, None, qk, qk, None, stream())
    torch.cuda.synchronize()
    c.close(view, c.want_forward(0), c.arithmetic())
