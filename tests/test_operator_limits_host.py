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


def test_calls_that_no_launch_can_hold_are_refused_before_anything_is_enqueued():
    # a matrix of 8192 x 1 has 512 pieces of 16 rows, a workgroup of 256 threads each: 2^32 threads from 32768 matrices on
    size, columns = P.ppll_orthogonalize_workspace_bytes, lambda n, at=0: P.matrix_group(at, 8192, 1, count=n)
    assert size([columns(32767)]) > 1 << 36
    small = P.matrix_group(0, 8, 8)
    for groups in ([columns(32768)], [columns(65535)], [columns(20000), columns(20000, 1 << 30)], [small, columns(32768, 64)],
                   [P.matrix_group(0, 2048, 2048, count=16384)]):
        with pytest.raises(P.PpllError) as e:
            size(groups)
        assert e.value.status == SHAPE
        for call in (lambda: P.ppll_orthogonalize(groups, P.FP32, 5, 16, 32, 48, 1 << 60),
                     lambda: P.ppll_muon_step(groups, 5, 16, 32, 48, None, 0.1, 0.9, True, 0.0, 64, 1 << 60)):
            with pytest.raises(P.PpllError) as e:
                call()
            assert e.value.status == SHAPE
