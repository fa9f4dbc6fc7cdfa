"""ResNet blocks with group norms in the place of BatchNorms, their inputs kept as they are or in 8 bits, against the float64 oracle: the operators
as a training step and an evaluation run them."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth
from helpers import assert_close, oracle_cfg, rel_l2
from test_gpu_parity import OUT_TOL, TOL, run_case

pytestmark = pytest.mark.gpu


def resnet(precision=synth.FP32, **more):
    wl = dict(arch=synth.RESNET, precision=precision, input_kind=synth.ACTIVATION, batch=4, num_classes=10, channels=16, height=6, width=6, n_basic_blocks=2,
              transition_block=0, aux_channels=24, img_c=3, optimizer=synth.SGD, momentum=0.9, nesterov=1, weight_decay=1e-4, bn_eps=1e-5, bn_momentum=0.1,
              lr=0.01, group_norm=4)
    wl.update(more)
    m = 2 if wl["transition_block"] else 1
    wl.update(img_h=m * wl["height"], img_w=m * wl["width"])
    return wl


CASES = [dict(), dict(input_kind=synth.IMAGE), dict(transition_block=2), dict(transition_block=1, input_kind=synth.IMAGE),
         dict(channels=12, aux_channels=20, height=5, width=7, batch=3), dict(group_norm=1, height=2, width=2), dict(group_norm=8, batch=1, n_basic_blocks=1)]


@pytest.mark.parametrize("case", CASES)
def test_fp32_steps(case):
    run_case(resnet(**case), 2, precision_floor=True)


BF16 = [dict(channels=32, height=16, width=16, batch=16), dict(n_basic_blocks=1), dict(input_kind=synth.IMAGE, n_basic_blocks=1, height=32, width=32),
        dict(transition_block=1, channels=32, n_basic_blocks=1, height=8, width=8), dict(channels=12, aux_channels=20, height=5, width=7, batch=3)]


@pytest.mark.parametrize("case", BF16)
@pytest.mark.parametrize("kept", [0, 1])
def test_bf16_steps(case, kept):
    run_case(resnet(synth.BF16, byte_checkpoints=kept, **case), 1)


@pytest.mark.parametrize("case", CASES)
def test_inputs_kept_in_bytes(case):
    """In fp32 a value near the middle between two bytes may fall to either side.  The products' sums are off by some 3e-6 of a row's largest
    element at the most, where a byte's step is 1/127 of that at the least: at most 2 * 3e-6 * 127 = 8e-4 of the bytes differ, each by a step, whose
    square is 12 times the mean square of what the rounding does to every element.  So gradients differ by sqrt(12 * 8e-4) = 0.1 of what keeping the
    inputs in bytes changes in them; held to 0.3 of it, tensor by tensor, and to the path's own tolerance."""
    from gpu_harness import GpuBlock
    wl = resnet(byte_checkpoints=1, **case)
    cfg = oracle_cfg(wl)
    flat = synth.make_params(O.param_spec(cfg), seed=1, jitter=True)
    st, plain = O.block_init(cfg, flat, np.float64), O.block_init(oracle_cfg(dict(wl, byte_checkpoints=0)), flat, np.float64)
    x, y = synth.make_batch(wl, seed=1)
    want_out, want_loss = O.block_step(st, x.astype(np.float64), y, 0.01)
    O.block_step(plain, x.astype(np.float64), y, 0.01)
    gb = GpuBlock(wl, flat)
    out, loss = gb.step(x, y, 0.01)
    grads = gb.tensors(P.T_GRAD)
    gb.close()
    assert abs(loss - want_loss) <= 1e-4 * abs(want_loss)
    assert_close(out, want_out, 1e-4, "x_out")
    for name, _ in O.param_spec(cfg):
        changed = rel_l2(plain.grads[name], st.grads[name])
        off = rel_l2(grads[name], st.grads[name])
        print(name, off, changed)
        assert off <= 1e-4 + 0.3 * changed, (name, off, changed)


@pytest.mark.parametrize("optimizer", [synth.ADAMW, synth.MUON])
def test_other_optimizers(optimizer):
    from test_gpu_block_options import muon_steps
    wl = resnet(optimizer=optimizer, lr=1e-3, beta1=0.9, beta2=0.999, adam_eps=1e-8, weight_decay=0.01)
    muon_steps(wl, 2) if optimizer == synth.MUON else run_case(wl, 1, precision_floor=True)


@pytest.mark.parametrize("precision", [synth.FP32, synth.BF16])
@pytest.mark.parametrize("kept", [0, 1])
@pytest.mark.parametrize("case", [dict(), dict(input_kind=synth.IMAGE, transition_block=2), dict(channels=12, aux_channels=20, height=5, width=7, batch=3)])
def test_evaluation_forwards(precision, case, kept):
    """The same values in both evaluation calls; those of a training step but for the order of fp32 roundings (its norms run in another kernel where
    they keep their inputs too): 2^-24 a rounding, of which a value passes some tens in each of seven layers at the most: 2e-5, beside bf16's 2^-8."""
    from gpu_harness import GpuBlock, to_device
    wl = resnet(precision, byte_checkpoints=kept, n_basic_blocks=2, **case)
    cfg = oracle_cfg(wl)
    flat = synth.make_params(O.param_spec(cfg), seed=5, jitter=True)
    gb = GpuBlock(wl, flat)
    st = O.block_init(cfg, flat, np.float64, storage="bf16" if precision == synth.BF16 else None)
    x, y = synth.make_batch(wl, seed=5)
    want_out, want = O.block_forward_eval(st, x.astype(np.float64))
    xd, got = to_device(x, wl), []
    for call in (P.ppll_block_forward_eval, P.ppll_block_forward_eval_noalloc):
        out, logits = torch.empty_like(gb.x_out), torch.empty(wl["batch"], 10, device="cuda:0")
        call(gb.h, xd, out, logits, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert_close(out.double().cpu().numpy(), want_out, OUT_TOL[precision], "x_out")
        assert_close(logits.double().cpu().numpy(), want, TOL[precision], "logits")
        got.append((out, logits))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    trained, _ = gb.step(x, y, 0.0)
    assert_close(trained, got[0][0].double().cpu().numpy(), 2e-5 if precision == synth.FP32 else 2.0 ** -8, "x_out of a training step")
    gb.close()


def test_a_block_without_running_statistics():
    from gpu_harness import GpuBlock
    wl = resnet()
    gb = GpuBlock(wl, synth.make_params(O.param_spec(oracle_cfg(wl)), seed=5))
    assert gb.bn(P.T_BN_MEAN) == {} and gb.bn(P.T_BN_VAR) == {}
    gb.close()


@pytest.mark.parametrize("kept", [0, 1])
def test_a_captured_step_is_replayed(kept):
    from gpu_harness import GpuBlock, to_device
    wl = resnet(synth.BF16, byte_checkpoints=kept, channels=32, height=16, width=16, batch=8, input_kind=synth.IMAGE)
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=9, jitter=True)
    block = GpuBlock(wl, flat)
    x, y = synth.make_batch(wl, seed=9)
    xd, yd = to_device(x, wl), torch.from_numpy(y.astype(np.int32)).to("cuda:0")
    step = lambda b: P.ppll_block_step(b.h, xd, yd, 0.002, b.x_out, b.loss, torch.cuda.current_stream().cuda_stream)  # noqa: E731
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(block)
    for _ in range(4):
        eager = GpuBlock(wl, flat)      # its first step starts its momentum as the captured one does
        for kind in (P.T_PARAM, P.T_MOMENT1):
            for i, (name, v) in enumerate(block.tensors(kind).items()):
                P.ppll_block_write_tensor(eager.h, kind, i, v)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(block.x_out, eager.x_out) and torch.equal(block.loss, eager.loss)
        for kind in (P.T_PARAM, P.T_MOMENT1, P.T_GRAD):
            a, b = block.tensors(kind), eager.tensors(kind)
            assert all(np.array_equal(a[n], b[n]) for n in a)
        eager.close()
    block.close()


def test_pipeline_equals_the_blocks_in_order():
    from test_gpu_pipeline import _run_pipeline, _run_sequential
    wls = [resnet(synth.BF16, input_kind=synth.IMAGE, byte_checkpoints=1, batch=8), resnet(synth.BF16, batch=8, n_basic_blocks=3)]
    flats = [synth.make_params(O.param_spec(oracle_cfg(w)), seed=j, jitter=True) for j, w in enumerate(wls)]
    batches = [synth.make_batch(wls[0], seed=1, index=i) for i in range(4)]
    got = _run_pipeline(wls, flats, batches, 2, 0.003)
    want = _run_sequential(wls, flats, batches, 0.003)
    assert np.array_equal(got[0], want[0])
    for a, b in zip(got[1], want[1]):
        assert all(np.array_equal(u, v) for u, v in zip(a, b))
