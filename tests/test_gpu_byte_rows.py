"""Rows of 8 bits, into and out of them, against the oracle: whole numbers, so equal."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from rows_helper import DEV, Placed, PlacedBytes, stream

pytestmark = pytest.mark.gpu
TYPES = [(P.FP32, torch.float32), (P.BF16, torch.bfloat16)]


def rows_of(rows, cols, dtype, seed=0):
    """Rows of very different size, one of zeros, some with values half way between two steps."""
    rng = np.random.default_rng([seed, rows, cols])
    x = rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-20, 20, (rows, 1)))
    x[rows // 2] = 0
    if rows > 2:
        x[0] = (rng.integers(-127, 127, cols) + 0.5) / 8
        x[0, 0] = 127 / 8
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def pack(precision, x, room=0, shift=0, out_room=0):
    rows, cols = x.shape
    src, out = Placed(x, x.dtype, room, shift), PlacedBytes(rows, cols, room=out_room)
    P.ppll_byte_rows_pack(precision, rows, cols, P.rows(src.view), P.byte_rows(out.store, out.exps), stream())
    return out


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (4, 15), (9, 16), (300, 17), (7, 33), (5, 64), (70, 100), (3, 129), (33, 200), (2, 256), (5, 500),
                                       (3, 513), (9, 1000), (3, 1536), (2, 2049), (3, 4097), (2, 8192), (2, 8200), (1, 20001)])
def test_pack(precision, dtype, rows, cols):
    x = rows_of(rows, cols, dtype)
    out = pack(precision, x)
    q, e = O.byte_rows(x.double().numpy())
    assert np.array_equal(out.e(), e) and np.array_equal(out.q(), q)
    assert out.padding_is_zero_and_the_rest_untouched()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("room,shift,out_room", [(1, 0, 16), (5, 3, 0), (8, 1, 32), (16, 8, 16)])
def test_pack_of_strided_rows(precision, dtype, room, shift, out_room):
    x = rows_of(37, 45, dtype, seed=1)
    out = pack(precision, x, room, shift, out_room)
    q, e = O.byte_rows(x.double().numpy())
    assert np.array_equal(out.e(), e) and np.array_equal(out.q(), q) and out.padding_is_zero_and_the_rest_untouched()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 8, 20, 40, 200, 3000, 9000])
def test_extremes(precision, dtype, cols):
    big = torch.finfo(dtype).max
    x = torch.zeros(9, cols)
    x[0, -1], x[1, 0], x[2, 0], x[3, -1] = float("nan"), float("inf"), -float("inf"), big
    x[4, 0], x[5, 0], x[6, -1], x[7, 0] = -big, 2.0 ** -126, -2.0 ** -127, 2.0 ** -133
    x = x.to(dtype)
    out = pack(precision, x)
    q, e = O.byte_rows(x.double().numpy())
    assert np.array_equal(out.e(), e) and np.array_equal(out.q(), q)
    assert out.e().tolist()[:3] == [-128] * 3
    back = Placed((9, cols), dtype)
    P.ppll_byte_rows_unpack(precision, 9, cols, P.byte_rows(out.store, out.exps), P.rows(back.view), stream())
    assert np.array_equal(back.host(), O.byte_values(q, e), equal_nan=True)


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows,cols,room,shift", [(1, 1, 0, 0), (5, 9, 3, 1), (70, 32, 0, 0), (9, 130, 1, 5), (3, 1000, 8, 8), (300, 17, 0, 3), (2, 9000, 0, 0)])
def test_unpack(precision, dtype, rows, cols, room, shift):
    q, e = O.byte_rows(rows_of(rows, cols, dtype, seed=2).double().numpy())
    src, out = PlacedBytes(rows, cols, q, e, room=16), Placed((rows, cols), dtype, room, shift)
    P.ppll_byte_rows_unpack(precision, rows, cols, P.byte_rows(src.store, src.exps), P.rows(out.view), stream())
    assert np.array_equal(out.host(), O.byte_values(q, e))
    assert out.untouched_around()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows,cols,room,shift", [(1, 1, 0, 0), (16, 32, 0, 0), (17, 33, 1, 3), (300, 40, 0, 0), (257, 8, 5, 1), (1000, 100, 4, 8), (5, 500, 0, 0), (64, 31, 0, 0)])
def test_pack_columns(precision, dtype, rows, cols, room, shift):
    x = rows_of(cols, rows, dtype, seed=3).t().contiguous()
    if cols > 3:
        x[rows // 3, 3] = float("nan")
    src, out = Placed(x, dtype, room, shift), PlacedBytes(cols, rows, room=16)
    P.ppll_byte_rows_pack_columns(precision, rows, cols, P.rows(src.view), P.byte_rows(out.store, out.exps), stream())
    q, e = O.byte_rows(x.double().numpy().T)
    assert np.array_equal(out.e(), e) and np.array_equal(out.q(), q) and out.padding_is_zero_and_the_rest_untouched()


@pytest.mark.parametrize("precision,dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(2048, 64), (2049, 65), (4096, 9), (4097, 20), (8192, 7), (9001, 130), (65536, 3)])
def test_pack_columns_of_many_rows(precision, dtype, rows, cols):
    """More rows than stay in registers, a last piece of one row, columns whose largest value is in the last or the first row."""
    x = rows_of(cols, rows, dtype, seed=4).t().contiguous()
    x[rows - 1, 0], x[0, 1] = 1e9, -1e9
    src, out = Placed(x, dtype), PlacedBytes(cols, rows, room=16)
    P.ppll_byte_rows_pack_columns(precision, rows, cols, P.rows(src.view), P.byte_rows(out.store, out.exps), stream())
    q, e = O.byte_rows(x.double().numpy().T)
    assert np.array_equal(out.e(), e) and np.array_equal(out.q(), q) and out.padding_is_zero_and_the_rest_untouched()


def test_rows_beyond_32_bits():
    # 70000 rows 32768 elements apart, columns of the last rows beyond 2^31 elements
    rows, cols, ld = 70000, 24, 32768
    store = torch.zeros(rows * ld, dtype=torch.bfloat16, device=DEV).view(rows, ld)
    x = store[:, -cols:]
    x.copy_(torch.randn(rows, cols, device=DEV))
    q, e = torch.empty(rows, 32, dtype=torch.int8, device=DEV), torch.empty(rows, dtype=torch.int8, device=DEV)
    P.ppll_byte_rows_pack(P.BF16, rows, cols, P.rows(x), P.byte_rows(q, e), stream())
    want_q, want_e = O.byte_rows(x[-500:].double().cpu().numpy())
    assert np.array_equal(q[-500:, :cols].cpu().numpy(), want_q) and np.array_equal(e[-500:].cpu().numpy(), want_e)
    x.zero_()
    P.ppll_byte_rows_unpack(P.BF16, rows, cols, P.byte_rows(q, e), P.rows(x), stream())
    assert np.array_equal(x[-500:].double().cpu().numpy(), O.byte_values(want_q, want_e))
    assert not bool(store[-1, :-cols].any())
