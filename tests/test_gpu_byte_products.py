"""ViT blocks whose encoder layers multiply rows of 8 bits, against the float64 oracle that rounds to the same rows: the operators as a training step
and an evaluation run them."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth
from helpers import oracle_cfg, rel_l2
from test_gpu_block_options import vit
from test_gpu_parity import TOL

pytestmark = pytest.mark.gpu


def block(precision=synth.FP32, **more):
    return vit(precision, **{**dict(rotary=0, qk_norm=0, byte_products=1), **more})


CASES = [dict(), dict(kind=synth.IMAGE), dict(aux=0, depth=1), dict(aux=2, depth=1), dict(rotary=1, qk_norm=1), dict(dim=60, heads=3, grid=(2, 2)),
         dict(dim=12, heads=6, grid=(1, 1), batch=3), dict(dim=66, heads=3, grid=(1, 7), mlp_dim=37), dict(kind=synth.IMAGE, batch=1, grid=(1, 1))]
# What the path's roundings do beside the rounding to bytes itself.  A value next to the middle between two bytes may fall to either side: by sums in
# fp32, off by some 3e-6 of a row's largest element at the most, at most 2 * 3e-6 * 127 = 8e-4 of the bytes, each by a step, whose square is 12 times
# the mean square of the rounding: sqrt(12 * 8e-4) = 0.1 of what the rounding changes in a result.  Values stored in bf16 are off by 2^-9 of
# themselves, some third of the row's largest: 127 / 3 * 2^-9 = 0.08 of a step, which moves 0.08 of the bytes to the next: sqrt(12 * 0.08) = 1.0 of it.
PART = {synth.FP32: 0.3, synth.BF16: 1.5}


def compare(wl, seed=1):
    from gpu_harness import GpuBlock
    cfg, lr = oracle_cfg(wl), wl["lr"]
    flat = synth.make_params(O.param_spec(cfg), seed=seed, jitter=True)
    st, plain = O.block_init(cfg, flat, np.float64), O.block_init(oracle_cfg(dict(wl, byte_products=0)), flat, np.float64)
    x, y = synth.make_batch(wl, seed=seed)
    want, want_loss = O.block_step(st, x.astype(np.float64), y, lr)
    other, other_loss = O.block_step(plain, x.astype(np.float64), y, lr)
    gb = GpuBlock(wl, flat)
    out, loss = gb.step(x, y, lr)
    grads, params = gb.tensors(P.T_GRAD), gb.tensors(P.T_PARAM)
    gb.close()
    tol, part = TOL[wl["precision"]], PART[wl["precision"]]
    assert abs(loss - want_loss) <= tol * abs(want_loss) + part * abs(other_loss - want_loss)
    report = [("x_out", rel_l2(out, want), rel_l2(other, want))]
    for n, shape in O.param_spec(cfg):
        g = st.grads[n].reshape(-1)
        if n.endswith(".qkv.b"):      # its middle third, the keys' bias, has a gradient of zero
            D = wl["dim"]
            keep = np.r_[0:D, 2 * D:3 * D]
            report.append((n, rel_l2(grads[n][keep], g[keep]), rel_l2(plain.grads[n][keep], g[keep])))
            continue
        report.append((n, rel_l2(grads[n], g), rel_l2(plain.grads[n], g)))
    print(*report, sep="\n")
    for n, off, changed in report:
        assert off <= tol + part * changed, (n, off, changed)
    # the update, from the gradients that the device has
    own = O.block_init(cfg, flat, np.float64)
    O.apply_update(own, {n: grads[n].reshape(s) for n, s in O.param_spec(cfg)}, lr)
    for n, _ in O.param_spec(cfg):
        assert rel_l2(params[n], own.params[n]) <= 1e-5
    return report


@pytest.mark.parametrize("case", CASES)
def test_fp32_steps(case):
    report = compare(block(**case))
    assert any(off < 0.5 * changed for _, off, changed in report)     # it is those rows that were multiplied


@pytest.mark.parametrize("case", [dict(dim=128, heads=2), dict(dim=128, heads=2, kind=synth.IMAGE, grid=(8, 8), batch=16), dict(dim=192, heads=3, grid=(6, 7)),
                                  dict(dim=96, heads=2, grid=(5, 3), rotary=1, qk_norm=1), dict(dim=66, heads=3, grid=(1, 7), mlp_dim=37)])
def test_bf16_steps(case):
    compare(block(synth.BF16, **case))


def test_with_muon():
    # the rule of the update alone: gradients are compared above
    from gpu_harness import GpuBlock
    wl = block(optimizer=synth.MUON, dim=64)
    cfg = oracle_cfg(wl)
    gb = GpuBlock(wl, synth.make_params(O.param_spec(cfg), seed=3, jitter=True))
    x, y = synth.make_batch(wl, seed=3)
    before = gb.tensors(P.T_PARAM)
    _, first = gb.step(x, y, 0.01)
    _, second = gb.step(x, y, 0.01)
    after = gb.tensors(P.T_PARAM)
    assert np.isfinite(first) and np.isfinite(second) and all(np.isfinite(after[n]).all() and (after[n] != before[n]).any() for n in after)
    gb.close()


@pytest.mark.parametrize("precision", [synth.FP32, synth.BF16])
@pytest.mark.parametrize("case", [dict(), dict(kind=synth.IMAGE, aux=0), dict(rotary=1, qk_norm=1, aux=2)])
def test_evaluation_forwards(precision, case):
    from gpu_harness import GpuBlock, to_device
    wl = block(precision, dim=128, heads=2, batch=5, **case)
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=5, jitter=True)
    gb = GpuBlock(wl, flat)
    x, y = synth.make_batch(wl, seed=5)
    got = []
    for call in (P.ppll_block_forward_eval, P.ppll_block_forward_eval_noalloc):
        out, logits = torch.empty_like(gb.x_out), torch.empty(5, 10, device="cuda:0")
        call(gb.h, to_device(x, wl), out, logits, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        got.append((out, logits))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    trained, _ = gb.step(x, y, 0.0)
    assert np.array_equal(trained, got[0][0].double().cpu().numpy())
    st = O.block_init(oracle_cfg(wl), flat, np.float64)
    plain = O.block_init(oracle_cfg(dict(wl, byte_products=0)), flat, np.float64)
    want, other = (O.block_forward_eval(s, x.astype(np.float64)) for s in (st, plain))
    for g, w, o in zip(got[0], want, other):
        assert rel_l2(g.double().cpu().numpy(), w) <= TOL[precision] + PART[precision] * rel_l2(o, w)
    gb.close()


def test_an_evaluation_leaves_the_activations_of_a_step():
    """Without an allocation: bytes of tokens and weights in the library's own buffer, not in the block's."""
    from gpu_harness import GpuBlock, to_device
    wl = block(synth.BF16, dim=128, heads=2, batch=5)
    gb = GpuBlock(wl, synth.make_params(O.param_spec(oracle_cfg(wl)), seed=5, jitter=True))
    x, y = synth.make_batch(wl, seed=5)
    gb.step(x, y, 0.0)
    torch.cuda.synchronize()
    before = gb.ws.clone()
    out, logits = torch.empty_like(gb.x_out), torch.empty(5, 10, device="cuda:0")
    P.ppll_block_forward_eval_noalloc(gb.h, to_device(x, wl), out, logits, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(before, gb.ws)
    gb.close()


def test_a_captured_step_is_replayed():
    from gpu_harness import GpuBlock, to_device
    wl = block(synth.BF16, dim=128, heads=2, kind=synth.IMAGE)
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=9, jitter=True)
    one = GpuBlock(wl, flat)
    x, y = synth.make_batch(wl, seed=9)
    xd, yd = to_device(x, wl), torch.from_numpy(y.astype(np.int32)).to("cuda:0")
    step = lambda b: P.ppll_block_step(b.h, xd, yd, 0.002, b.x_out, b.loss, torch.cuda.current_stream().cuda_stream)  # noqa: E731
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(one)
    for _ in range(4):
        eager = GpuBlock(wl, flat)      # its first step starts its momentum as the captured one does
        for kind in (P.T_PARAM, P.T_MOMENT1):
            for i, (name, v) in enumerate(one.tensors(kind).items()):
                P.ppll_block_write_tensor(eager.h, kind, i, v)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(one.x_out, eager.x_out) and torch.equal(one.loss, eager.loss)
        for kind in (P.T_PARAM, P.T_MOMENT1, P.T_GRAD):
            a, b = one.tensors(kind), eager.tensors(kind)
            assert all(np.array_equal(a[n], b[n]) for n in a)
        eager.close()
    one.close()


def test_pipeline_equals_the_blocks_in_order():
    from test_gpu_pipeline import _run_pipeline, _run_sequential
    base = dict(dim=128, heads=2, batch=8, lr=0.003)
    wls = [block(synth.BF16, kind=synth.IMAGE, aux=1, **base), block(synth.BF16, aux=1, byte_products=0, **base), block(synth.BF16, aux=0, **base)]
    flats = [synth.make_params(O.param_spec(oracle_cfg(w)), seed=j, jitter=True) for j, w in enumerate(wls)]
    batches = [synth.make_batch(wls[0], seed=1, index=i) for i in range(4)]
    got = _run_pipeline(wls, flats, batches, 2, 0.003)
    want = _run_sequential(wls, flats, batches, 0.003)
    assert np.array_equal(got[0], want[0])
    for a, b in zip(got[1], want[1]):
        assert all(np.array_equal(u, v) for u, v in zip(a, b))
