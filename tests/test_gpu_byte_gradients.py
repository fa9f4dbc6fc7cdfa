"""Gradients of linear layers on rows of 8 bits at the ends of their ranges: dX of more elements than one product addresses."""
import pytest
import torch

from paper_2411_12780_amd import binding as P
from rows_helper import DEV, stream
from test_gpu_byte_linear import ULP, Layer, check_backward

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
