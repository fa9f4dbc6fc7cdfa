"""cos and sin of the rotation, seen through pairs (1, 0), which come out as (cos, sin)."""
import numpy as np
import pytest
import torch

from paper_2411_12780_amd import binding as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def turned(positions, pairs, base):
    """cos and sin [positions, pairs] in fp32 as the kernel takes them, and the angles in 64 bits."""
    tokens = len(positions)
    x = torch.zeros(tokens, 2 * pairs, device=DEV)
    x[:, :pairs] = 1
    cfg = P.rotary_config(P.FP32, tokens, tokens, 1, 0, 2 * pairs, [pairs], base)
    qk = P.queries_keys(x, None)
    P.ppll_qk_rotary_forward(cfg, torch.from_numpy(positions.astype(np.int32)).to(DEV), None, None, qk, qk, None, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    got = x.double().cpu().numpy()
    return got[:, :pairs], got[:, pairs:], positions[:, None].astype(np.float64) * np.float64(np.float32(base)) ** (-np.arange(pairs) / pairs)


@pytest.mark.parametrize("pairs", [16, 17])      # pieces of heads, and element by element
def test_cos_and_sin_are_off_by_their_own_roundings(pairs):
    # The functions of an fp32 argument are off by up to 3/4 of a unit in the last place (the last sum of their series half a unit, what is before it half of
    # that), the correction for the argument's rounding rounds once more, by half a unit at most; errors spread evenly: 0.52 units in the mean.  Over a
    # circle a unit is 5.04e-8 in the mean: 2.6e-8, and a tenth of slack.  An argument rounded to 32 bits alone costs 3.2e-8 with exact functions.
    rng = np.random.default_rng(pairs)
    cos, sin, angle = turned(rng.integers(-(1 << 20), 1 << 20, 30000), pairs, 3.0)
    for got, want in ((cos, np.cos(angle)), (sin, np.sin(angle))):
        assert np.sqrt(np.mean((got - want) ** 2)) <= 2.9e-8


@pytest.mark.parametrize("base", [0.01, 0.5, 1.0, 100.0])
@pytest.mark.parametrize("pairs", [16, 17])
def test_far_positions_of_every_base(base, pairs):
    # roundings of 2^-53 on the way to a turn, relative: exponent 3 of its |log2|, 2 to 4 of the power, the quotient by 2 pi and the product; in the oracle here
    # one of the exponent's and 2 more.  Those of cos and sin themselves are 2^-23 at most.
    positions = np.random.default_rng(2).integers(-(1 << 31), 1 << 31, 4000)
    cos, sin, angle = turned(positions, pairs, base)
    octaves = abs(np.log2(np.float64(np.float32(base)))) * np.arange(pairs) / pairs
    limit = np.abs(angle) * (6 + 4 * octaves) * 2.0 ** -53 + 2.0 ** -23
    for got, want in ((cos, np.cos(angle)), (sin, np.sin(angle))):
        assert (np.abs(got - want) <= limit).all()
