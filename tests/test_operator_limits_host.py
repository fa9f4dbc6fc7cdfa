"""Many layers, many matrices, and what lies at the limits of the orthogonalised updates: host arithmetic only, no call here launches."""
import random
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


def elements(g):
    """Of a group: for each of its matrices, all side by side being one, the first element, one past the last, columns from the first."""
    if g.count > 1 and g.stride < (g.rows - 1) * g.ld + g.cols:
        cols = [i * g.stride + c for i in range(g.count) for c in range(g.cols)]
        return [(g.offset, g.offset + (g.rows - 1) * g.ld + cols[-1] + 1, cols)]
    return [(g.offset + i * g.stride, g.offset + i * g.stride + (g.rows - 1) * g.ld + g.cols, list(range(g.cols))) for i in range(g.count)]


def by_the_rule(x, y):
    """Extents that overlap need one ld and different columns of it."""
    for la, ha, ca in elements(x):
        for lb, hb, cb in elements(y):
            if la < hb and lb < ha and (x.ld != y.ld or {c % x.ld for c in ca} & {(lb - la + c) % x.ld for c in cb}):
                return False
    return True


def touched(g):
    at = [g.offset + i * g.stride + r * g.ld + c for i in range(g.count) for r in range(g.rows) for c in range(g.cols)]
    assert len(set(at)) == len(at)
    return set(at)


def test_what_is_shared_is_refused_and_what_is_not_is_taken():
    rng = random.Random(5)
    taken = refused = beside = 0
    for _ in range(6000):
        ld = rng.randint(4, 14)
        pair = []
        for _ in range(2):
            rows, cols = rng.randint(1, 4), rng.randint(1, 4)
            mine = ld if rng.random() < 0.8 else rng.randint(4, 14)
            extent = (rows - 1) * mine + cols
            if rng.random() < 0.5:                           # side by side
                stride = rng.randint(cols, cols + 4)
                count = rng.randint(1, max(1, (mine - cols) // stride + 1))
            else:
                stride, count = extent + rng.choice([0, 1, rng.randint(0, 60)]), rng.randint(1, 6)
            pair.append(P.matrix_group(rng.randint(0, 90), rows, cols, ld=mine, count=count, stride=stride))
        want = by_the_rule(*pair)
        try:
            P.ppll_orthogonalize_workspace_bytes(pair)
            got = True
        except P.PpllError:
            got = False
        assert got == want, [[getattr(g, f) for f, _ in g._fields_] for g in pair]
        if got:
            assert not touched(pair[0]) & touched(pair[1])
            taken += 1
            beside += any(a < d and c < b for a, b, _ in elements(pair[0]) for c, d, _ in elements(pair[1]))
        else:
            refused += 1
    assert taken > 1000 and refused > 1000 and beside > 50


def test_groups_side_by_side_that_take_turns_are_taken():
    # query and key parts of three heads in one weight, a head's query beside its key
    group = lambda at: P.matrix_group(at, 8, 4, ld=24, count=3, stride=8)  # noqa: E731
    assert P.ppll_orthogonalize_workspace_bytes([group(0), group(4)]) == 0


def test_many_matrices_are_compared_in_microseconds():
    # groups apart, parts of weights that take turns, and small matrices within one stride of one another
    far = [P.matrix_group((i << 33), 30, 30, count=65535, stride=901) for i in range(16)]
    parts = [P.matrix_group(i * 40, 40, 40, ld=640, count=65535, stride=25600) for i in range(16)]
    between = [P.matrix_group(i * 16, 4, 4, count=65535, stride=4000) for i in range(16)]
    for groups in (far, parts, between):
        # a walk over all matrices of each of the 120 pairs takes 24 to 120 ms
        assert min(seconds(P.ppll_orthogonalize_workspace_bytes, groups) for _ in range(5)) < 5e-3


@pytest.mark.parametrize("dk", [4096, 4096 + 28, 4096 - 28])
def test_gradients_of_the_two_scales_that_share_memory_are_refused(dk):
    for rows in (8, 0):
        cfg = P.rotary_config(P.FP32, rows, 4, 2, 1, 8, [2, 2], 100.0)
        qk = P.QueriesKeys(16, 32, 16, 8)
        with pytest.raises(P.PpllError) as e:
            P.ppll_qk_rotary_backward(cfg, 16, 16, 16, qk, qk, qk, 4096, dk, 64, P.ppll_qk_rotary_workspace_bytes(cfg))
        assert e.value.status == SHAPE and "scales" in P.ppll_last_error()


def test_many_matrices_between_many_columns_are_compared_as_quickly():
    # 65535 columns side by side, and as many matrices of one element between them, whichever group comes first
    columns = P.matrix_group(0, 2, 1, ld=1 << 20, count=65535, stride=16)
    between = P.matrix_group(8, 1, 1, ld=1 << 20, count=65535, stride=16)
    for groups in ([columns, between], [between, columns]):
        assert min(seconds(P.ppll_orthogonalize_workspace_bytes, groups) for _ in range(2)) < 0.1
