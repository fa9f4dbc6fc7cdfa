"""ResNet blocks with group norms in the place of BatchNorms, on the CPU: what is refused, what older callers get, workspaces, and the oracle's
gradients against differences."""
import ctypes

import numpy as np
import pytest

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth
from helpers import oracle_cfg

GOOD = synth.workload("resnet_stage_bf16", batch=4, group_norm=8)
OLD = P.BlockConfig.group_norm.offset
size = lambda wl: P.ppll_block_workspace_bytes(P.make_config(wl))  # noqa: E731


@pytest.mark.parametrize("bad", [dict(group_norm=-1), dict(group_norm=7), dict(group_norm=64), dict(group_norm=32, channels=32, transition_block=2),
                                 dict(aux_channels=20), dict(aux_channels=4104), dict(byte_checkpoints=2), dict(byte_checkpoints=-1),
                                 dict(group_norm=0, byte_checkpoints=1), dict(bn_eps=float("inf")), dict(bn_eps=float("nan")), dict(bn_eps=0.0),
                                 dict(reserved=1), dict(byte_products=1)])
def test_refused_resnet_configurations(bad):
    with pytest.raises(P.PpllError) as e:
        size(dict(GOOD, **bad))
    assert e.value.status == 2


@pytest.mark.parametrize("bad", [dict(group_norm=8), dict(byte_checkpoints=1), dict(reserved=1), dict(byte_products=2), dict(byte_products=-1),
                                 dict(byte_products=1, mlp_dim=65537), dict(byte_products=1, dim=21848, heads=8)])
def test_refused_vit_configurations(bad):
    with pytest.raises(P.PpllError) as e:
        size(synth.workload("vit_tiny_fp32", **bad))
    assert e.value.status == 2


@pytest.mark.parametrize("name", ["vit_tiny_fp32", "vit_stage_muon_bf16", "resnet_stage_bf16"])
def test_configurations_that_end_in_front_of_the_new_fields_are_taken(name):
    wl = synth.workload(name)
    cfg = P.make_config(wl)
    cfg.struct_size = OLD
    cfg.group_norm = cfg.byte_checkpoints = cfg.reserved = 77       # memory behind the caller's structure
    assert P.ppll_block_workspace_bytes(cfg) == size(wl)


@pytest.mark.parametrize("bytes_", [OLD - 4, OLD + 4, ctypes.sizeof(P.BlockConfig) - 4])
def test_other_sizes_are_refused(bytes_):
    cfg = P.make_config(GOOD)
    cfg.struct_size = bytes_
    with pytest.raises(P.PpllError) as e:
        P.ppll_block_workspace_bytes(cfg)
    assert e.value.status == 2


def test_inputs_kept_in_bytes_take_less_memory():
    wl = dict(GOOD, batch=128)
    maps = 10 * 128 * 16 * 16 * 32                # elements that the norms of five basic blocks read
    # in the place of 2 bytes an element: 1 byte and 1/32 for the exponent; one map of full width for the next product's output
    assert size(wl) - size(dict(wl, byte_checkpoints=1)) >= maps * (2 - 1 - 1 / 32) - 2 * maps / 10 - (1 << 20)


def test_products_in_bytes_take_less_memory():
    wl = synth.workload("vit_stage_act_bf16")
    M, D, F, layers = wl["batch"] * wl["tokens"], wl["dim"], wl["mlp_dim"], wl["depth"] + wl["aux_depth"]
    # for all layers but one, what the products read, in 2 bytes an element: the norms' outputs (2 D wide) and the MLP's middle (F); and gradients of 4 D + F
    # that wait for a launch at the end.  In their place a byte, and one of attention's output (D), that attention's backward keeps as it is too
    layers -= 1                                   # the auxiliary network's last layer stays as it is
    saved = (layers - 1) * M * (2 * (2 * D + F) + 2 * (4 * D + F) - (3 * D + F))
    weights = layers * (4 * D * D + 2 * D * F)
    assert size(wl) - size(dict(wl, byte_products=1)) >= 0.5 * saved - weights > 0


def test_there_are_no_running_statistics():
    assert O.bn_stat_spec(oracle_cfg(GOOD)) == []
    assert [n for n, _ in O.param_spec(oracle_cfg(GOOD))] == [n for n, _ in O.param_spec(oracle_cfg(dict(GOOD, group_norm=0)))]


@pytest.mark.parametrize("case", [dict(), dict(transition_block=1, height=3, width=4), dict(input_kind=synth.IMAGE, img_h=5, img_w=4, img_c=3)])
def test_gradients_of_the_oracle_are_differences_of_its_loss(case):
    wl = dict(synth.workload("resnet_stage_bf16", batch=2, channels=8, height=5, width=4, n_basic_blocks=2, aux_channels=12, group_norm=4), **case)
    cfg = oracle_cfg(wl)
    flat = synth.make_params(O.param_spec(cfg), seed=2, jitter=True).astype(np.float64)
    x, y = synth.make_batch(wl, seed=2)

    def loss(values):
        st = O.block_init(cfg, values, np.float64)
        return O.cross_entropy(O.resnet_forward(st, x)[1], y)[0]
    st = O.block_init(cfg, flat, np.float64)
    _, logits, caches = O.resnet_forward(st, x)
    g = O.resnet_backward(st, O.cross_entropy(logits, y)[1], caches)
    rng, off, checked = np.random.default_rng(4), 0, 0
    for name, shape in O.param_spec(cfg):
        n = int(np.prod(shape))
        i = int(rng.integers(n))
        h = 1e-6
        lo, hi = flat.copy(), flat.copy()
        lo[off + i] -= h
        hi[off + i] += h
        d = (loss(hi) - loss(lo)) / (2 * h)
        # a difference of losses of order one at 2^-53 over 2e-6, and h^2 of the third derivative; a ReLU that changes within h breaks it,
        # which so few pixels do not meet but by chance
        assert abs(d - g[name].reshape(-1)[i]) <= 1e-7 + 1e-6 * abs(d), name
        off += n
        checked += 1
    assert checked == len(g)
