"""Many layers, many matrices, and what lies at the limits of the orthogonalised updates: host arithmetic only, no call here launches."""
import time

import pytest

from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth

CONFIG, SHAPE = 2, 3
DEEP = synth.workload("vit_stage_muon_bf16", batch=1, dim=8, heads=1, mlp_dim=16, aux_depth=1)


def seconds(call, *args):
    start = time.perf_counter()
    call(*args)
    return time.perf_counter() - start


def test_a_deep_block_is_planned_in_time_that_grows_with_its_layers():
    # 30000 layers have 180000 matrices and 360000 tensors: half a second, and half a minute if each tensor is compared with each matrix
    size = lambda n: P.ppll_block_workspace_bytes(P.make_config(dict(DEEP, depth=n)))  # noqa: E731
    assert size(30000) > 9 * size(3000)
    assert seconds(size, 30000) < 5


def test_a_block_whose_matrices_are_too_many_for_one_call_is_refused():
    cfg = P.make_config(dict(DEEP, depth=65534, dim=1536, heads=24, mlp_dim=8192))
    for call in (P.ppll_block_workspace_bytes, P.ppll_block_param_bytes, lambda c: P.ppll_pipeline_workspace_bytes([c], 1)):
        with pytest.raises(P.PpllError) as e:
            call(cfg)
        assert e.value.status == CONFIG and "too many matrices" in P.ppll_last_error()
