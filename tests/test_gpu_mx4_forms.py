"""The forms that large aligned models take, against the definition: vector accesses of every type in messages and operands, the model step beside them,
and sums of errors over more parts than a warp adds up."""
import numpy as np
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from tests import _mx4
from tests.test_gpu_mx4 import DT, Case, bits, same

pytestmark = pytest.mark.gpu
# every layer starts on 32 bytes and has whole groups of eight blocks; the last ones end inside a group and inside a block
ALIGNED = [256 * 5, 32768 * 2 + 512, 8, 40000, 256, 1000, 32 * 9 + 16, 24]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("W", [1, 3])
def test_step_of_aligned_layers(dtype, W):
    c = Case(ALIGNED, W, 0, dtype, seed=W)
    assert c.stride % 8 == 0 and c.grads.data_ptr() % 32 == 0 and c.state.data_ptr() % 32 == 0
    for _ in range(2):
        want = c.expect()
        kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
        torch.cuda.synchronize()
        c.check(*want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_absent_blocks_of_aligned_layers(dtype):
    c = Case(ALIGNED, 2, 0, dtype, hard=False)
    c.grads[0, 700], c.grads[1, 1280 + 4000], c.grads[1, 1280 + 32768 + 31] = float("nan"), float("inf"), -float("inf")
    want = c.expect()
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    torch.cuda.synchronize()
    c.check(*want)
    assert (c.msg.scales.cpu().numpy() == 255).sum() == 3
    est = torch.full_like(c.state, 7.0)
    kb.kimad_mx4_apply(c.ctx, c.msg, est)
    for w in range(2):
        _, _, v, gone, _ = want[0][w]
        assert np.array_equal(est[w].cpu().numpy(), np.where(gone, np.float32(7), np.float32(7) + v.astype(np.float32)))


@pytest.mark.parametrize("layers,dtype", [([32768 * 20 + 5, 100, 33], "f32"), ([32768 * 20 + 5, 100, 33], "bf16"), ([100, 32768 * 17, 32768 * 40 + 8, 3000], "f16")])
def test_errors_of_layers_of_many_parts_in_one_launch(layers, dtype):
    """Few chunks, so the pass adds the errors up itself; sixteen parts a chunk, so the large layers have more than 256 of them."""
    c = Case(layers, 1, 0, dtype)
    launches = kb.kimad_launch_count(c.ctx)
    want = c.expect()
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    torch.cuda.synchronize()
    assert kb.kimad_launch_count(c.ctx) == launches + 1
    c.check(*want)


@pytest.mark.parametrize("W", [1, 2, 3, 8])
def test_model_step_over_aligned_layers(W):
    """Bit for bit by the definition: estimators, then sum over the senders in their order, then the model."""
    c = Case(ALIGNED, W, 0, hard=False, seed=W)
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    c.msg.scales[0, 2] = 255
    values = torch.zeros_like(c.state)
    kb.kimad_mx4_read(c.ctx, c.msg, values)
    g = torch.Generator(device="cuda").manual_seed(3)
    est, x = torch.randn((W, c.N), device="cuda", generator=g), torch.randn(c.N, device="cuda", generator=g)
    assert est.data_ptr() % 32 == 0 and x.data_ptr() % 32 == 0
    weights, gamma = [np.float32((m + 1) / 70) for m in range(W)], np.float32(0.3)
    want, v = est.cpu().numpy(), values.cpu().numpy()
    gone = np.zeros((W, c.N), bool)
    gone[0, 64:96] = True
    want = np.where(gone, want, want + v)
    acc = np.zeros(c.N, np.float32)
    for m in range(W):
        acc = acc + weights[m] * want[m]
    model = x.cpu().numpy() - gamma * acc
    est2, x2 = est.clone(), x.clone()
    kb.kimad_mx4_apply(c.ctx, c.msg, est, x, weights, gamma)
    kb.kimad_mx4_apply(c.ctx, c.msg, est2)
    kb.kimad_aggregate(x2, est2, weights, gamma)
    torch.cuda.synchronize()
    assert np.array_equal(bits(est), want.view(np.uint32)) and np.array_equal(bits(x), model.view(np.uint32))
    assert torch.equal(est, est2) and torch.equal(x, x2)


@pytest.mark.parametrize("along", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pad", [(256, 1024, 0), (128, 2304, 8), (384, 5632, 0), (130, 1280, 2), (256, 1024, 1), (1024, 768, 0)])
def test_operands_of_whole_tiles(rows, cols, pad, dtype, along):
    """Whole tiles and whole lines of 1024 values, with rows on vectors (pad 0, 8), on pairs (2) and on neither (1)."""
    v = _mx4.hard_values((rows, cols), np.random.default_rng(rows + cols))
    v = np.clip(v, -60000, 60000) if dtype == "f16" else v
    v[3, 5], v[-1, 40] = np.nan, np.inf
    room = torch.full((rows, cols + pad), 3.0, dtype=DT[dtype], device="cuda")
    x = room[:, :cols]
    x.copy_(torch.from_numpy(v))
    v = x.float().cpu().numpy()
    lines, length = (cols, rows) if along == 0 else (rows, cols)
    op = kb.Mx4Operand(lines, length)
    kb.kimad_mx4_quantize(x, op, along)
    c, t, values = _mx4.operand(np.ascontiguousarray(v.T if along == 0 else v))
    values = values.T if along == 0 else values
    backs = [torch.full((rows, cols + pad), 3.0, dtype=d, device="cuda") for d in (torch.float32, torch.bfloat16)]
    for b in backs:
        kb.kimad_mx4_dequantize(op, b[:, :cols], along)
    torch.cuda.synchronize()
    assert np.array_equal(op.codes.cpu().numpy().reshape(lines, -1), c) and np.array_equal(op.scales.cpu().numpy().reshape(-1), t.reshape(-1))
    for b in backs:
        assert same(b[:, :cols].double().cpu().numpy(), values) and (b[:, cols:] == 3.0).all()
    assert (room[:, cols:] == 3.0).all()
