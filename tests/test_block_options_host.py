"""Configurations with rotary positions, normalised queries and keys and the Muon optimizer: what is refused, what older callers get."""
import ctypes

import pytest

from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth
from host_hip import calls, compile_runtime

GOOD = synth.workload("vit_stage_muon_bf16", depth=1)
OLD = P.BlockConfig.rotary.offset       # size of a configuration before those fields


@pytest.mark.parametrize("bad", [dict(rotary=2), dict(qk_norm=-1), dict(grid_h=7), dict(grid_h=4, grid_w=16), dict(grid_h=0, grid_w=0), dict(rotary_base=0.0),
                                 dict(rotary_base=-1.0), dict(rotary_base=float("inf")), dict(rotary_base=float("nan")), dict(qk_norm_eps=0.0),
                                 dict(qk_norm_eps=float("nan")), dict(heads=128), dict(heads=1), dict(mlp_dim=8200),
                                 dict(input_kind=synth.ACTIVATION, grid_h=65536, grid_w=65536), dict(optimizer=3), dict(depth=65535, aux_depth=1)])
def test_refused_vit_configurations(bad):
    with pytest.raises(P.PpllError) as e:
        P.ppll_block_workspace_bytes(P.make_config(dict(GOOD, **bad)))
    assert e.value.status == 2


@pytest.mark.parametrize("bad", [dict(rotary=1), dict(qk_norm=1), dict(optimizer=synth.MUON, channels=912), dict(optimizer=synth.MUON, aux_channels=8200), dict(optimizer=synth.MUON, n_basic_blocks=65536)])
def test_refused_resnet_configurations(bad):
    with pytest.raises(P.PpllError) as e:
        P.ppll_block_workspace_bytes(P.make_config(synth.workload("resnet_stage_bf16", batch=1, **bad)))
    assert e.value.status == 2


def test_a_mlp_of_any_width_without_muon():
    assert P.ppll_block_workspace_bytes(P.make_config(dict(GOOD, mlp_dim=8200, optimizer=synth.ADAMW, batch=1))) > 0


def old(wl):
    """The same configuration as a caller passes it that was built before the new fields; behind it, memory that is not zero."""
    cfg = P.make_config(wl)
    cfg.struct_size = OLD
    for f in ("rotary", "grid_h", "grid_w", "qk_norm"):
        setattr(cfg, f, 77)
    return cfg


@pytest.mark.parametrize("name", ["vit_tiny_fp32", "vit_stage_bf16", "resnet_stage_bf16"])
def test_configurations_without_the_new_fields_are_taken(name):
    wl = synth.workload(name)
    for size in (P.ppll_block_workspace_bytes, P.ppll_block_param_bytes, P.ppll_block_in_bytes, P.ppll_block_out_bytes):
        assert size(old(wl)) == size(P.make_config(wl))


@pytest.mark.parametrize("size", [0, OLD - 8, OLD + 4, ctypes.sizeof(P.BlockConfig) + 8])
def test_other_sizes_are_refused(size):
    cfg = P.make_config(synth.workload("vit_tiny_fp32"))
    cfg.struct_size = size
    with pytest.raises(P.PpllError) as e:
        P.ppll_block_workspace_bytes(cfg)
    assert e.value.status == 2


def test_a_pipeline_of_older_configurations():
    # they lie closer together than the present ones
    wls = [synth.workload("vit_stage_bf16"), synth.workload("vit_stage_act_bf16")]
    raw = b"".join(bytes(old(w))[:OLD] for w in wls)
    buf = ctypes.create_string_buffer(raw, len(raw))
    n = ctypes.c_size_t(0)
    call = P.lib().ppll_pipeline_workspace_bytes
    assert call(ctypes.cast(buf, ctypes.POINTER(P.BlockConfig)), 2, 2, ctypes.byref(n)) == 0
    assert n.value == P.ppll_pipeline_workspace_bytes([P.make_config(w) for w in wls], 2)


def test_a_pipeline_takes_one_size_of_configurations():
    mixed = [P.make_config(synth.workload("vit_stage_bf16")), old(synth.workload("vit_stage_act_bf16"))]
    with pytest.raises(P.PpllError) as e:
        P.ppll_pipeline_workspace_bytes(mixed, 2)
    assert e.value.status == 2


def test_a_workspace_holds_the_update_and_the_kept_queries():
    size = lambda **more: P.ppll_block_workspace_bytes(P.make_config(dict(GOOD, **more)))  # noqa: E731
    plain = size(optimizer=synth.ADAMW, rotary=0, grid_h=0, grid_w=0, qk_norm=0)
    turned = size(optimizer=synth.ADAMW, qk_norm=0)
    assert plain < turned <= plain + 65 * 2 * 4 + 4096
    assert size(optimizer=synth.ADAMW) >= turned + 2 * 128 * 65 * 384 * 2      # queries and keys of the first layer
    assert size() > size(optimizer=synth.ADAMW)


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    exe = compile_runtime(str(tmp_path_factory.mktemp("runtime")))
    return lambda workloads, *what: calls(exe, workloads, *what)


@pytest.mark.parametrize("name", ["vit_stage_bf16", "resnet_stage_bf16", "vit_tiny_fp32"])
def test_blocks_without_the_options_launch_none_of_it(runtime, name):
    (made,) = runtime([synth.workload(name)], "step")
    kernels = [c[5] for c in made if c[0] == "launch"]
    assert not any(part in k for k in kernels for part in ("rotary", "product_kernel", "normalise", "adamw_ranges"))


def test_launches_of_a_block_with_the_options(runtime):
    made, evaluated = runtime([GOOD], "step", "eval")
    kernels = [c[5] for c in made if c[0] == "launch"]
    # one layer and a pruned auxiliary one, whose queries are the class token's: three forward, three backward
    assert sum("rotary" in k for k in kernels) == 6
    assert sum("adamw_ranges" in k for k in kernels) == 1 and not any("adamw_kernel" in k for k in kernels)
    assert sum("rotary" in c[5] for c in evaluated if c[0] == "launch") == 3
