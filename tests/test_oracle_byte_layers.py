"""Pins of the oracle's rows of 8 bits and group norm: closed forms, torch.autograd, differences."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O

TORCH_ACT = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}


def test_byte_rows_of_known_rows():
    x = np.array([[127.0, -1.0, 0.5, 1.5, 2.5], [128.0, 1.0, 3.0, -5.0, 0.0], [0, 0, 0, 0, 0], [np.nan, 1, 2, 3, 4], [1, -np.inf, 2, 3, 4],
                  [2.0 ** -130, 0, 0, 0, 0], [3.4e38, -3.4e38, 1, 0, 0]])
    q, e = O.byte_rows(x)
    assert e.tolist() == [0, 1, -126, -128, -128, -126, 121]
    assert q[0].tolist() == [127, -1, 0, 2, 2]             # ties to even
    assert q[1].tolist() == [64, 0, 2, -2, 0]              # 0.5, 1.5 and -2.5 to even
    assert not q[2:6].any() and q[6].tolist() == [127, -127, 0, 0, 0]
    v = O.byte_values(q, e)
    assert v[0, 0] == 127 and v[1, 0] == 128 and np.isnan(v[3:5]).all() and v[6, 0] == 127 * 2.0 ** 121


def test_byte_rows_are_within_half_a_step_that_is_no_larger_than_needed():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 30)) * np.exp(rng.uniform(-40, 40, (200, 1)))
    q, e = O.byte_rows(x)
    assert (np.abs(O.byte_values(q, e) - x) <= 2.0 ** (e[:, None] - 1)).all()
    assert (np.abs(q).max(1) >= 63).all() and (np.abs(q).max(1) <= 127).all()


@pytest.mark.parametrize("act", list(TORCH_ACT))
@pytest.mark.parametrize("groups,channels", [(1, 6), (3, 6), (6, 6)])
def test_group_norm_against_autograd(act, groups, channels):
    rng = np.random.default_rng([1, groups])
    x, res, dy = (rng.standard_normal((2, 5, channels)) for _ in range(3))
    g, b = 1 + 0.3 * rng.standard_normal(channels), 0.3 * rng.standard_normal(channels)
    t = [torch.tensor(a, requires_grad=True) for a in (x, res, g, b)]
    n = torch.nn.functional.group_norm(t[0].transpose(1, 2), groups, t[2], t[3], 1e-3).transpose(1, 2)
    y = TORCH_ACT[act](n + t[1])
    y.backward(torch.tensor(dy))
    mine, stats, z = O.group_norm_fwd(x, g, b, groups, 1e-3, act, res)
    dz = dy * O.activation(act, z)[1]
    dx, dg, db = O.group_norm_bwd(dz, x, stats, g)
    for a, ref in ((mine, y.detach()), (dx, t[0].grad), (dz, t[1].grad), (dg, t[2].grad), (db, t[3].grad)):
        assert np.allclose(a, ref.numpy(), atol=1e-12)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_by_differences(act):
    z, h = np.linspace(-6, 6, 101), 1e-5
    up, down = O.activation(act, z + h)[0], O.activation(act, z - h)[0]
    assert np.allclose(O.activation(act, z)[1], (up - down) / (2 * h), atol=1e-9)
