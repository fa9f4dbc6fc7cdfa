"""What the calls on rows of 8 bits and group norm refuse, on the host: no call here gets as far as a launch."""
import ctypes
import math

import pytest
import torch

from paper_2411_12780_amd import binding as P

NULL, CONFIG, SHAPE, WORKSPACE = 1, 2, 3, 4
BIG = 1 << 50


def refused(status, call, *args):
    with pytest.raises(P.PpllError) as e:
        call(*args)
    assert e.value.status == status, (e.value, args)
    assert P.ppll_last_error()


def R(p=4096, ld=64):
    return P.Rows(p, ld)


def B(q=8192, e=4096, ld=64):
    return P.ByteRows(q, e, ld)


@pytest.mark.parametrize("call,sides", [(P.ppll_byte_rows_pack, (R, B)), (P.ppll_byte_rows_unpack, (B, R)), (P.ppll_byte_rows_pack_columns, (R, B))])
def test_rows_refusals(call, sides):
    columns = call is P.ppll_byte_rows_pack_columns

    def go(precision=P.BF16, rows=60, cols=60, plain=R(), eight=B()):
        call(precision, rows, cols, *((plain, eight) if sides[0] is R else (eight, plain)))

    for status, bad in ((CONFIG, dict(precision=2)), (CONFIG, dict(precision=-1)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=65537)), (SHAPE, dict(rows=(1 << 30) + 1)),
                        (NULL, dict(plain=None)), (NULL, dict(plain=R(p=None))), (NULL, dict(eight=None)), (NULL, dict(eight=B(q=None))), (NULL, dict(eight=B(e=None))),
                        (SHAPE, dict(plain=R(p=4097))), (SHAPE, dict(plain=R(p=4098), precision=P.FP32)), (SHAPE, dict(plain=R(ld=59))), (SHAPE, dict(plain=R(ld=1 << 31))),
                        (SHAPE, dict(eight=B(q=8200))), (SHAPE, dict(eight=B(ld=48))), (SHAPE, dict(eight=B(ld=72))), (SHAPE, dict(eight=B(ld=(1 << 20) + 16)))):
        refused(status, lambda: go(**bad))
    if columns:
        refused(SHAPE, lambda: go(rows=0))
        refused(SHAPE, lambda: go(rows=65537))
        go(cols=0, plain=None, eight=None)            # nothing to do
    else:
        refused(SHAPE, lambda: go(cols=0))
        go(rows=0, plain=None, eight=None)


GOOD = dict(precision=P.BF16, rows=100, in_dim=60, out_dim=60)


@pytest.mark.parametrize("bad", [dict(precision=2), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(in_dim=0), dict(out_dim=0), dict(in_dim=65537), dict(out_dim=65537),
                                 dict(activation=P.ACT_RELU), dict(activation=P.ACT_SILU), dict(activation=4), dict(activation=-1),
                                 dict(rows=1 << 30, in_dim=65536), dict(rows=1 << 30, out_dim=65536)])
def test_linear_configurations_that_are_refused(bad):
    refused(CONFIG, P.ppll_byte_linear_workspace_bytes, P.byte_linear_config(**{**GOOD, **bad}))


def test_linear_refusals():
    refused(NULL, P.ppll_byte_linear_workspace_bytes, None)
    cfg = P.byte_linear_config(**GOOD)
    cfg.struct_size = 8
    refused(CONFIG, P.ppll_byte_linear_workspace_bytes, cfg)
    cfg = P.byte_linear_config(**GOOD)
    assert P.lib().ppll_byte_linear_workspace_bytes(ctypes.byref(cfg), None) == NULL
    gelu = P.byte_linear_config(**GOOD, activation=P.ACT_GELU)
    forward = lambda c=cfg, x=B(), w=B(), bias=16, res=None, y=R(), slope=None: P.ppll_byte_linear_forward(c, x, w, bias, res, y, slope)  # noqa: E731
    for status, bad in ((NULL, dict(x=None)), (NULL, dict(w=None)), (NULL, dict(y=None)), (NULL, dict(c=None)), (SHAPE, dict(bias=18)), (SHAPE, dict(res=R(ld=59))),
                        (SHAPE, dict(res=R(p=4097))), (NULL, dict(res=R(p=None))), (SHAPE, dict(y=R(ld=59))), (SHAPE, dict(x=B(ld=48))), (SHAPE, dict(w=B(q=8193))),
                        (CONFIG, dict(slope=R())), (SHAPE, dict(c=gelu, slope=R(ld=1))), (NULL, dict(c=gelu, slope=R(p=None)))):
        refused(status, lambda: forward(**bad))
    wide = P.byte_linear_config(P.BF16, 60000, 128, 128)
    need = P.ppll_byte_linear_workspace_bytes(wide)
    assert need > 0 and need % 4 == 0
    back = lambda c=wide, x=B(ld=128), w=B(ld=128), dy=R(ld=128), gate=None, dx=R(ld=128), dw=64, db=64, ws=64, n=need: P.ppll_byte_linear_backward(  # noqa: E731
        c, x, w, dy, gate, dx, dw, db, ws, n)
    for status, bad in ((NULL, dict(c=None)), (NULL, dict(x=None)), (NULL, dict(w=None)), (NULL, dict(dy=None)), (NULL, dict(dx=None, gate=R())), (SHAPE, dict(dw=66)),
                        (SHAPE, dict(db=66)), (NULL, dict(ws=None)), (WORKSPACE, dict(ws=72)), (WORKSPACE, dict(n=need - 1)), (SHAPE, dict(dx=R(ld=100))),
                        (SHAPE, dict(gate=R(ld=100))), (SHAPE, dict(dy=R(ld=100))), (SHAPE, dict(x=B(ld=112)))):
        refused(status, lambda: back(**bad))
    P.ppll_byte_linear_backward(wide, None, None, None, None, None, None, None)      # nothing wanted
    none = P.byte_linear_config(P.BF16, 0, 60, 60)
    assert P.ppll_byte_linear_workspace_bytes(none) == 0
    P.ppll_byte_linear_forward(none, None, None, None, None, None)


NORM = dict(precision=P.BF16, images=3, pixels=20, channels=60, groups=4)


@pytest.mark.parametrize("bad", [dict(precision=2), dict(images=-1), dict(pixels=0), dict(images=1 << 20, pixels=1 << 11), dict(channels=0, groups=1), dict(channels=4097, groups=1),
                                 dict(groups=0), dict(groups=7), dict(groups=-4), dict(activation=4), dict(activation=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf),
                                 dict(eps=math.nan)])
def test_norm_configurations_that_are_refused(bad):
    refused(CONFIG, P.ppll_group_norm_workspace_bytes, P.group_norm_config(**{**NORM, **bad}))


def test_norm_refusals():
    refused(NULL, P.ppll_group_norm_workspace_bytes, None)
    cfg = P.group_norm_config(**NORM)
    cfg.struct_size = 8
    refused(CONFIG, P.ppll_group_norm_workspace_bytes, cfg)
    cfg, relu, silu = (P.group_norm_config(**NORM, activation=a) for a in (P.ACT_NONE, P.ACT_RELU, P.ACT_SILU))
    need = P.ppll_group_norm_workspace_bytes(cfg)
    assert need > 0
    forward = lambda c=cfg, x=R(), g=64, b=64, res=None, y=R(), st=None, keep=None, ws=64, n=need: P.ppll_group_norm_forward(c, x, g, b, res, y, st, keep, ws, n)  # noqa: E731
    for status, bad in ((NULL, dict(c=None)), (NULL, dict(x=None)), (NULL, dict(g=None)), (NULL, dict(b=None)), (NULL, dict(y=None)), (SHAPE, dict(g=66)), (SHAPE, dict(b=66)),
                        (SHAPE, dict(st=66)), (SHAPE, dict(x=R(ld=59))), (SHAPE, dict(y=R(p=4097))), (SHAPE, dict(res=R(ld=59))), (NULL, dict(res=R(p=None))),
                        (SHAPE, dict(keep=B(ld=48))), (NULL, dict(keep=B(e=None))), (NULL, dict(ws=None)), (WORKSPACE, dict(ws=72)), (WORKSPACE, dict(n=need - 1))):
        refused(status, lambda: forward(**bad))
    back = lambda c=cfg, x=R(), x8=None, st=64, g=64, b=64, res=None, y=None, dy=R(), dx=R(8192), dr=None, dg=1024, db=2048, ws=64, n=need: (  # noqa: E731
        P.ppll_group_norm_backward(c, x, x8, st, g, b, res, y, dy, dx, dr, dg, db, ws, n))
    for status, bad in ((NULL, dict(c=None)), (NULL, dict(x=None)), (SHAPE, dict(x8=B())), (SHAPE, dict(x=None, x8=B(ld=48))), (NULL, dict(st=None)), (NULL, dict(g=None)),
                        (NULL, dict(b=None)), (NULL, dict(dy=None)), (NULL, dict(dx=None)), (NULL, dict(dg=None)), (NULL, dict(db=None)), (SHAPE, dict(dg=1026)),
                        (SHAPE, dict(dg=2048)), (SHAPE, dict(dg=2048 + 236)), (NULL, dict(c=relu)), (SHAPE, dict(c=relu, y=R(ld=1))), (SHAPE, dict(c=silu, res=R(ld=1))),
                        (SHAPE, dict(dr=R(8192))), (SHAPE, dict(dr=R(ld=1))), (NULL, dict(ws=None)), (WORKSPACE, dict(n=need - 1)), (WORKSPACE, dict(ws=72))):
        refused(status, lambda: back(**bad))
    none = P.group_norm_config(**{**NORM, "images": 0})
    P.ppll_group_norm_forward(none, None, None, None, None, None)
    refused(NULL, lambda: back(c=none, dg=None))


def test_outputs_that_are_inputs():
    gelu = P.byte_linear_config(**GOOD, activation=P.ACT_GELU)
    forward = lambda **k: P.ppll_byte_linear_forward(gelu, B(), B(), 16, k.get("res"), R(4096), k.get("slope"))  # noqa: E731
    refused(SHAPE, lambda: forward(res=R(4096, 72)))
    refused(SHAPE, lambda: forward(slope=R(4096)))
    refused(SHAPE, lambda: forward(res=R(8192), slope=R(8192)))
    cfg = P.byte_linear_config(**GOOD)
    need = P.ppll_byte_linear_workspace_bytes(cfg)
    refused(SHAPE, lambda: P.ppll_byte_linear_backward(cfg, B(), B(), R(4096), None, R(4096), 64, 64, 64, need))
    refused(SHAPE, lambda: P.ppll_byte_linear_backward(cfg, B(), B(), R(4096), R(8192, 72), R(8192), 64, 64, 64, need))
    cfg = P.group_norm_config(**NORM)
    need = P.ppll_group_norm_workspace_bytes(cfg)
    refused(SHAPE, lambda: P.ppll_group_norm_forward(cfg, R(4096, 72), 64, 64, None, R(4096), None, None, 64, need))
    refused(SHAPE, lambda: P.ppll_group_norm_forward(cfg, R(8192), 64, 64, R(4096, 72), R(4096), None, None, 64, need))
    back = lambda x=R(4096), dy=R(8192), dx=R(16384), dr=None: P.ppll_group_norm_backward(cfg, x, None, 64, 64, 64, None, None, dy, dx, dr, 1024, 2048, 64, need)  # noqa: E731
    for bad in (dict(dx=R(4096)), dict(dx=R(8192, 72)), dict(dr=R(8192, 72)), dict(dr=R(4096)), dict(dr=R(16384))):
        refused(SHAPE, lambda: back(**bad))


def test_tensors_of_rows():
    refused(SHAPE, P.rows, torch.zeros(2, 3, 4))
    refused(SHAPE, P.rows, torch.zeros(4, 3).t())
    assert P.rows(torch.zeros(6, 9)[:, 3:7]).ld == 9
    q, e = torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, dtype=torch.int8)
    assert P.byte_rows(q, e).ld == 32 and P.byte_rows(q[:, :20], e).ld == 32
    refused(SHAPE, P.byte_rows, q.float(), e)
    refused(SHAPE, P.byte_rows, q, e.float())
    refused(SHAPE, P.byte_rows, q, torch.zeros(8, dtype=torch.int8)[::2])
