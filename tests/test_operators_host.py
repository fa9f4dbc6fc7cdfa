"""What the operators' entry points refuse, on the host: no call here gets as far as a launch."""
import ctypes
import math

import pytest

from paper_2411_12780_amd import binding as P

NULL, CONFIG, SHAPE, WORKSPACE = 1, 2, 3, 4


def refused(status, call, *args):
    with pytest.raises(P.PpllError) as e:
        call(*args)
    assert e.value.status == status, (e.value, args)
    assert P.ppll_last_error()


def test_workspace_of_groups():
    size = P.ppll_orthogonalize_workspace_bytes
    assert size([]) == 0
    assert size([P.matrix_group(0, 8, 8, count=0)]) == 0
    assert size([P.matrix_group(0, 8, 8, count=1000)]) == 0        # small ones never leave their workgroup
    one = size([P.matrix_group(0, 300, 400)])
    assert one > 0 and one % 256 == 0
    assert size([P.matrix_group(0, 300, 400), P.matrix_group(120000, 300, 400)]) > one
    assert size([P.matrix_group(0, 8192, 8192)]) >= 8192 * 8192 * 4


@pytest.mark.parametrize("group", [
    dict(offset=0, rows=0, cols=4), dict(offset=0, rows=4, cols=0), dict(offset=0, rows=8193, cols=4), dict(offset=0, rows=4, cols=8193),
    dict(offset=-1, rows=4, cols=4), dict(offset=0, rows=4, cols=4, ld=3), dict(offset=0, rows=4, cols=4, count=-1),
    dict(offset=0, rows=4, cols=4, count=65536), dict(offset=0, rows=4, cols=4, count=2, stride=15),
    dict(offset=0, rows=4, cols=4, count=2, stride=0), dict(offset=0, rows=4, cols=4, count=2, stride=-16),
    dict(offset=0, rows=4, cols=4, ld=8, count=3, stride=4),         # side by side, but the third leaves the row
    dict(offset=0, rows=4, cols=4, ld=9, count=2, stride=3),         # side by side, sharing a column
    dict(offset=1 << 41, rows=4, cols=4)])
def test_groups_that_are_refused(group):
    refused(SHAPE, P.ppll_orthogonalize_workspace_bytes, [P.matrix_group(**group)])


def test_groups_that_share_elements_are_refused():
    size, g = P.ppll_orthogonalize_workspace_bytes, P.matrix_group
    qkv = [g(i * 4, 4, 4, ld=12, count=3, stride=100) for i in range(3)]
    assert size(qkv) == 0                                           # query, key and value parts of three layers
    assert size([g(0, 4, 4, ld=12, count=3, stride=4), g(48, 4, 8)]) == 0
    refused(SHAPE, size, [g(0, 4, 4), g(0, 4, 4)])                  # the same twice
    refused(SHAPE, size, [g(0, 4, 4), g(15, 2, 2)])
    refused(SHAPE, size, [g(0, 4, 5, ld=12), g(4, 4, 4, ld=12)])    # a common column
    refused(SHAPE, size, [g(0, 4, 4, ld=12), g(10, 4, 4, ld=12)])   # columns 10..13 are 10, 11 and 0, 1 of the next row
    refused(SHAPE, size, [g(0, 4, 4, ld=12), g(4, 4, 4, ld=11)])    # interleaved with another row length
    refused(SHAPE, size, [g(0, 4, 4, count=10, stride=100), g(715, 2, 2)])      # the eighth matrix is 700..715
    assert size([g(0, 4, 4, count=10, stride=100), g(716, 2, 2)]) == 0
    assert size([g(0, 4, 4, count=10, stride=100), g(715, 2, 2, count=0)]) == 0
    assert size([g(0, 4, 4, count=10, stride=100), g(16, 4, 4, count=10, stride=100), g(32, 4, 4, count=5, stride=200)]) == 0


def test_more_groups_than_a_call_takes():
    groups = [P.matrix_group(16 * i, 4, 4) for i in range(17)]
    refused(SHAPE, P.ppll_orthogonalize_workspace_bytes, groups)
    assert P.ppll_orthogonalize_workspace_bytes(groups[:16]) == 0
    g = P.MatrixGroup(0, 16, 4, 4, 4, 1, 1)                         # reserved
    refused(SHAPE, P.ppll_orthogonalize_workspace_bytes, [g])
    n = ctypes.c_size_t(0)
    assert P.lib().ppll_orthogonalize_workspace_bytes(None, 1, ctypes.byref(n)) == NULL
    assert P.lib().ppll_orthogonalize_workspace_bytes((P.MatrixGroup * 1)(g), -1, ctypes.byref(n)) == SHAPE
    assert P.lib().ppll_orthogonalize_workspace_bytes((P.MatrixGroup * 1)(P.matrix_group(0, 4, 4)), 1, None) == NULL


def test_orthogonalize_refusals():
    g = [P.matrix_group(0, 300, 300)]
    ws = P.ppll_orthogonalize_workspace_bytes(g)
    call = P.ppll_orthogonalize
    refused(CONFIG, call, g, 2, 5, 16, 16, 16, ws)
    refused(CONFIG, call, g, P.FP32, 0, 16, 16, 16, ws)
    refused(CONFIG, call, g, P.FP32, 17, 16, 16, 16, ws)
    refused(NULL, call, g, P.FP32, 5, None, 16, 16, ws)
    refused(NULL, call, g, P.FP32, 5, 16, None, 16, ws)
    refused(NULL, call, g, P.FP32, 5, 16, 16, None, ws)
    refused(WORKSPACE, call, g, P.FP32, 5, 24, 16, 16, ws)
    refused(WORKSPACE, call, g, P.FP32, 5, 16, 24, 16, ws)
    refused(WORKSPACE, call, g, P.FP32, 5, 16, 16, 24, ws)
    refused(WORKSPACE, call, g, P.FP32, 5, 16, 16, 16, ws - 1)
    call([], P.FP32, 5, None, None, None, 0)                        # nothing to do


def test_muon_refusals():
    g = [P.matrix_group(0, 300, 300)]
    ws = P.ppll_orthogonalize_workspace_bytes(g)
    def call(steps=5, grads=16, m=32, p=48, shadow=None, lr=0.1, momentum=0.9, decay=0.0, work=64, nbytes=ws):
        P.ppll_muon_step(g, steps, grads, m, p, shadow, lr, momentum, True, decay, work, nbytes)
    for status, bad in ((CONFIG, dict(steps=0)), (CONFIG, dict(lr=math.nan)), (CONFIG, dict(momentum=math.nan)), (CONFIG, dict(decay=math.nan)),
                        (NULL, dict(grads=None)), (NULL, dict(m=None)), (NULL, dict(p=None)), (NULL, dict(work=None)),
                        (WORKSPACE, dict(grads=8)), (WORKSPACE, dict(m=8)), (WORKSPACE, dict(p=8)), (WORKSPACE, dict(shadow=8)),
                        (WORKSPACE, dict(nbytes=ws - 1)), (SHAPE, dict(grads=32)), (SHAPE, dict(m=48)), (SHAPE, dict(shadow=48)), (SHAPE, dict(shadow=16))):
        refused(status, lambda: call(**bad))


GOOD = dict(precision=P.FP32, rows=8, tokens=4, q_heads=2, k_heads=1, head_dim=8, pairs=[2, 2], base=100.0)


@pytest.mark.parametrize("bad", [
    dict(precision=2), dict(rows=-4), dict(rows=7), dict(tokens=0), dict(q_heads=-1), dict(q_heads=0, k_heads=0), dict(q_heads=65537),
    dict(head_dim=7), dict(head_dim=0), dict(head_dim=258), dict(pairs=[3, 2]), dict(pairs=[-1, 2]), dict(base=0.0),
    dict(base=-1.0), dict(base=math.inf), dict(base=math.nan)])
def test_rotary_configurations_that_are_refused(bad):
    refused(CONFIG, P.ppll_qk_rotary_workspace_bytes, P.rotary_config(**{**GOOD, **bad}))


def test_rotary_refusals():
    cfg = P.rotary_config(**GOOD)
    ws = P.ppll_qk_rotary_workspace_bytes(cfg)
    assert ws > 0
    refused(CONFIG, lambda: P.rotary_config(**{**GOOD, "pairs": []}))
    refused(CONFIG, lambda: P.rotary_config(**{**GOOD, "pairs": [1, 1, 1, 1]}))
    refused(NULL, P.ppll_qk_rotary_workspace_bytes, None)
    small = P.rotary_config(**GOOD)
    small.struct_size = 8
    refused(CONFIG, P.ppll_qk_rotary_workspace_bytes, small)
    axes = P.rotary_config(**GOOD)
    axes.axes = 4
    refused(CONFIG, P.ppll_qk_rotary_workspace_bytes, axes)
    qk = lambda q=16, k=16, ql=16, kl=8: P.QueriesKeys(q, k, ql, kl)  # noqa: E731
    forward = lambda c=cfg, pos=16, qs=None, ks=None, x=qk(), y=qk(), keep=None: P.ppll_qk_rotary_forward(c, pos, qs, ks, x, y, keep)  # noqa: E731
    for status, bad in ((NULL, dict(pos=None)), (SHAPE, dict(pos=18)), (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(x=qk(q=None))),
                        (NULL, dict(y=qk(k=None))), (SHAPE, dict(x=qk(q=18))), (SHAPE, dict(x=qk(ql=15))), (SHAPE, dict(y=qk(kl=7))),
                        (SHAPE, dict(keep=qk(ql=15))), (NULL, dict(qs=16)), (NULL, dict(ks=16)), (SHAPE, dict(qs=16, ks=18)),
                        (SHAPE, dict(x=qk(ql=1 << 40)))):
        refused(status, lambda: forward(**bad))
    for eps in (0.0, -1.0, math.nan):
        refused(CONFIG, lambda: forward(c=P.rotary_config(**GOOD, norm_eps=eps), qs=16, ks=16))
    back = lambda qs=16, ks=16, x=qk(), dy=qk(), dx=qk(), dq=16, dk=16, w=16, n=ws: P.ppll_qk_rotary_backward(  # noqa: E731
        cfg, 16, qs, ks, x, dy, dx, dq, dk, w, n)
    for status, bad in ((NULL, dict(x=None)), (NULL, dict(dy=None)), (NULL, dict(dx=None)), (NULL, dict(dq=None)), (NULL, dict(dk=None)),
                        (SHAPE, dict(dq=18)), (NULL, dict(w=None)), (WORKSPACE, dict(w=24)), (WORKSPACE, dict(n=ws - 1)), (NULL, dict(ks=None))):
        refused(status, lambda: back(**bad))
    none = P.rotary_config(**{**GOOD, "rows": 0})
    P.ppll_qk_rotary_forward(none, None, None, None, None, None)      # no rows: nothing to do
    P.ppll_qk_rotary_backward(none, None, None, None, None, None, None)


def test_sides_are_two_dimensional_rows():
    import torch
    refused(SHAPE, P.queries_keys, torch.zeros(2, 3, 4), None)
    refused(SHAPE, P.queries_keys, torch.zeros(4, 3).t(), None)
    s = P.queries_keys(None, torch.zeros(6, 9)[:, 3:7])
    assert s.k_ld == 9 and s.q is None
