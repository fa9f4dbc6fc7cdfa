"""That ViT blocks with byte_products in bf16 multiply the rows of 8 bits, and not the bf16 values that those were made from.

bf16 storage blurs single results as much as the rounding to bytes changes them, but not which way they go.  With `plain` the float64 oracle without
byte_products, c = (oracle with them) - plain and d = device - plain, the share <d, c> / <c, c> says how much of that change the device has: 0
where it multiplies something else (its own roundings know nothing of c: off by |roundings| / |c| / sqrt(elements), 1 / sqrt(2000) at the most here), 1 where
both sides make the same bytes.  Between a value's rounding errors on both sides, d of a step apart, lies (1 - 6 |d| + 6 d^2) of their square.
  Stored in bf16 a value is off by 2^-9 of itself at the most, half of that on average; values are a third of a row's largest, 20 to 40 steps:
  |d| = 0.03, a share of 0.8, and 0.03 of the bytes are others: sqrt(12 * 0.03) = 0.6 of the rounding's effect.
  A product behind another one takes values that those bytes have moved: the rounding is 0.29 of a step, 0.7 % of such a value, so the product is
  off by 0.6 * 0.7 % = 0.4 % of itself, 0.17 of a step in the next rounding (0.14 on average): a share of 1 - 0.84 + 0.17 = 0.33.
  Weights are in fp32, their bytes are the same: a share of 1 of what they change.
So the line between bytes and none is drawn at 1/4, under all of these and ten deviations over 0, and at 3/2 above."""
import numpy as np
import pytest
import torch

from oracle import ppll_oracle as O
from paper_2411_12780_amd import binding as P
from paper_2411_12780_amd import synth
from helpers import oracle_cfg, rel_l2
from test_gpu_byte_products import block
from test_gpu_orthogonalize import bound

pytestmark = pytest.mark.gpu
CASES = [dict(dim=128, heads=2, depth=1, aux=0), dict(dim=128, heads=2, depth=1, aux=1), dict(dim=192, heads=3, grid=(6, 7), depth=1, aux=0),
         dict(dim=96, heads=2, grid=(5, 3), depth=1, aux=0, rotary=1, qk_norm=1), dict(dim=128, heads=2, depth=1, aux=0, kind=synth.IMAGE, grid=(8, 8)),
         dict(dim=66, heads=3, grid=(5, 7), mlp_dim=37, depth=1, aux=0)]
BIG = dict(batch=24)


def share(device, with_bytes, plain):
    c = (with_bytes - plain).reshape(-1)
    return float((device - plain).reshape(-1) @ c / (c @ c))


def oracles(wl, flat):
    return [O.block_init(oracle_cfg(dict(wl, byte_products=b)), flat, np.float64) for b in (1, 0)]


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("byte_products", [1, 0])
def test_steps(case, byte_products):
    # (the block without them shows that the share would see it)
    from gpu_harness import GpuBlock
    wl = block(synth.BF16, **{**BIG, **case})
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=31, jitter=True)
    x, y = synth.make_batch(wl, seed=31)
    states = oracles(wl, flat)
    (want, _), (plain, _) = (O.block_step(st, x.astype(np.float64), y, wl["lr"]) for st in states)
    gb = GpuBlock(dict(wl, byte_products=byte_products), flat)
    out, _ = gb.step(x, y, wl["lr"])
    grads = gb.tensors(P.T_GRAD)
    gb.close()
    shares = {"x_out": share(out, want, plain)}
    # gradients of the layer's four products, forward and backward behind them
    for name in ("blk0.qkv.w", "blk0.proj.w", "blk0.fc1.w", "blk0.fc2.w"):
        shares[name] = share(grads[name], *(st.grads[name].reshape(-1) for st in states))
    print(shares)
    assert all(0.25 < v < 1.5 if byte_products else v < 0.25 for v in shares.values()), shares


@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("byte_products", [1, 0])
def test_evaluations(case, byte_products):
    from gpu_harness import GpuBlock, to_device
    wl = block(synth.BF16, **{**BIG, **case})
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=32, jitter=True)
    x, _ = synth.make_batch(wl, seed=32)
    (want, _), (plain, _) = (O.block_forward_eval(st, x.astype(np.float64)) for st in oracles(wl, flat))
    gb = GpuBlock(dict(wl, byte_products=byte_products), flat)
    for call in (P.ppll_block_forward_eval, P.ppll_block_forward_eval_noalloc):
        out = torch.empty_like(gb.x_out)
        call(gb.h, to_device(x, wl), out, None, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        v = share(out.double().cpu().numpy(), want, plain)
        print(v)
        assert 0.25 < v < 1.5 if byte_products else v < 0.25
    gb.close()


@pytest.mark.parametrize("precision", [synth.FP32, synth.BF16])
def test_muon_updates(precision):
    """The rule of the update on the block's own gradients, within what the orthogonalisation's roundings come to (see `bound`)."""
    from gpu_harness import GpuBlock
    wl = block(precision, optimizer=synth.MUON, dim=128, heads=2)
    cfg = oracle_cfg(wl)
    spec = O.param_spec(cfg)
    flat = synth.make_params(spec, seed=33, jitter=True)
    x, y = synth.make_batch(wl, seed=33)
    gb = GpuBlock(wl, flat)
    gb.step(x, y, wl["lr"])
    grads, params, own = gb.tensors(P.T_GRAD), gb.tensors(P.T_PARAM), O.block_init(cfg, flat, np.float64)
    gb.close()
    O.apply_update(own, {n: grads[n].reshape(s) for n, s in spec}, wl["lr"])
    for name, shape in spec:
        most = 1e-5
        if O.is_hidden_matrix(name):
            g = grads[name].reshape(-1, shape[-1])
            u = g * (1 + wl["momentum"] if wl["nesterov"] else 1)
            off = sum((0.2 * max(part.shape) ** 0.5 * bound(part, 5) * np.linalg.norm(O.orthogonalize(part))) ** 2
                      for part in np.split(u, 3 if name.endswith(".qkv.w") else 1, axis=1)) ** 0.5
            most += wl["lr"] * off / np.linalg.norm(own.params[name])
        assert rel_l2(params[name], own.params[name]) <= most, name


@pytest.mark.parametrize("precision", [synth.FP32, synth.BF16])
@pytest.mark.parametrize("size", [dict(dim=128, heads=2, depth=2, aux=0, batch=24), dict(dim=66, heads=3, grid=(5, 7), mlp_dim=37, depth=1, aux=0, batch=24),
                                  dict(dim=768, heads=12, depth=1, aux=0, grid=(15, 16), batch=64, mlp_dim=2304)])
def test_launch_brackets_count_the_products_of_bytes(precision, size):
    """Forward, input and weight gradient of the four products of each layer, 2 M N K each, and the same results with the brackets as without."""
    from gpu_harness import GpuBlock
    wl = block(precision, **size)
    flat = synth.make_params(O.param_spec(oracle_cfg(wl)), seed=34, jitter=True)
    x, y = synth.make_batch(wl, seed=34)
    losses = []
    for on in (False, True):
        gb = GpuBlock(wl, flat)
        P.ppll_block_profile_enable(gb.h, on)
        losses.append(gb.step(x, y, 0.01)[1])
        ms, flops, n = P.ppll_block_profile_read(gb.h)
        P.ppll_block_profile_enable(gb.h, False)
        gb.close()
        M, D, F = wl["batch"] * wl["tokens"], wl["dim"], wl["mlp_dim"]
        forward = wl["depth"] * 2.0 * M * (D * 3 * D + D * D + 2 * D * F)
        if on:
            assert n >= 8 * wl["depth"] and ms > 0 and abs(flops - 3 * forward) <= 1e-6 * flops, (n, ms, flops, 3 * forward)
        else:
            assert n == 0
    assert losses[0] == losses[1]
