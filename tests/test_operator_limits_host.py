"""Many layers, many matrices, and what lies at the limits of the orthogonalised updates: host arithmetic only, no call here launches."""
import time

from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth

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
