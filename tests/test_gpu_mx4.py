"""4-bit messages and operands on the GPU against their definition in 64 bits.  Codes, scales, states and values are compared bit for bit; sums of
squares within half a step of binary32 for the one rounding at the end, and as much again for the order of the binary64 sums."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from paper_2312_08053_b200 import workloads
from tests import _mx4
from tests._harness import Runner

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LAYERS = {
    "one": [1],
    "edges": [1, 31, 32, 33, 255, 256, 257, 7, 64],
    "chunks": [5, 32768 * 2 + 5, 100, 40000, 32640, 1],
    "many": [3] * 700 + [64] * 200,
    "large": [40000 * 257, 9, 32768 * 300, 33] + [40000] * 40 + [100] * 900,  # more than 1184 chunks: the errors by a kernel of their own
}


def bits(t):
    return t.cpu().numpy().view(np.uint32)


def same(a, b):
    """Equal values and equal zeros' signs, NaN in the same places."""
    a, b = np.asarray(a), np.asarray(b)
    return a.shape == b.shape and np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(np.where(np.isnan(a), 0, a), np.where(np.isnan(b), 0, b)) \
        and np.array_equal(np.signbit(a[~np.isnan(a)]), np.signbit(b[~np.isnan(b)]))


class Case:
    """A context and inputs; grads may start `shift` elements into their buffer, rows may be longer than N."""

    def __init__(self, layers, W, pad=0, dtype="f32", shift=0, seed=0, hard=True, **opts):
        self.layers, self.W, self.N = layers, W, sum(layers)
        self.stride = self.N + pad
        self.ctx = kb.new_context(layers, W, [1.0], D=max(1000, len(layers)), worker_stride=self.stride, **opts)
        self.msg = kb.Mx4Message(self.ctx)
        rng = np.random.default_rng(seed)
        make = _mx4.hard_values if hard else (lambda s, r: r.standard_normal(s).astype(np.float32))
        g = make((W, self.stride), rng)
        buf = torch.zeros(W * self.stride + shift, dtype=DT[dtype], device="cuda")
        self.grads = buf[shift:].view(W, self.stride)
        if dtype == "f16":
            g = np.clip(g, -60000, 60000)
        self.grads.copy_(torch.from_numpy(g))
        sbuf = torch.zeros(W * self.stride + shift, device="cuda")
        self.state = sbuf[shift:].view(W, self.stride)
        self.state.copy_(torch.from_numpy(make((W, self.stride), rng) * np.float32(0.25)))

    def expect(self):
        g, s = self.grads.float().cpu().numpy(), self.state.cpu().numpy()
        with np.errstate(over="ignore", invalid="ignore"):
            d = g - s
            out = [_mx4.message(d[w, :self.N], self.layers) for w in range(self.W)]
            new = s.copy()
            for w, (_, _, v, gone, _) in enumerate(out):
                new[w, :self.N] = np.where(gone, s[w, :self.N], s[w, :self.N] + v.astype(np.float32))
        return out, new

    def check(self, out, new):
        codes, scales, err = self.msg.codes.cpu().numpy(), self.msg.scales.cpu().numpy(), self.msg.err.cpu().numpy()
        st = self.msg.stats_host()
        blocks = sum(-(-n // 32) for n in self.layers)
        for w, (c, sc, _, gone, e) in enumerate(out):
            assert np.array_equal(codes[w], c)
            assert np.array_equal(scales[w, :blocks], sc)
            with np.errstate(over="ignore"):
                want = e.astype(np.float32)
                total = np.float32(e.sum())
            fine = np.isfinite(want)
            assert np.array_equal(fine, np.isfinite(err[w]))
            assert np.allclose(err[w][fine].astype(np.float64), e[fine], rtol=2.0 ** -23, atol=2.0 ** -149)
            assert np.allclose(float(st["total_err"][w]), float(total), rtol=2.0 ** -23)
            assert int(st["used_bytes"][w]) == 17 * blocks and int(st["n_selected"][w]) == self.N and int(st["budget_bytes"][w]) == 0
        assert np.array_equal(bits(self.state), new.view(np.uint32))
        assert kb.kimad_debug_check(self.ctx)[1:] == (0, 0)


@pytest.mark.parametrize("layers,W,pad,dtype,shift", [
    ("one", 1, 0, "f32", 0), ("one", 3, 1, "bf16", 1), ("edges", 1, 0, "f32", 0), ("edges", 2, 0, "f32", 1), ("edges", 3, 5, "f16", 3),
    ("chunks", 1, 0, "f32", 0), ("chunks", 2, 0, "bf16", 0), ("chunks", 2, 3, "f32", 2), ("many", 2, 0, "f32", 0), ("many", 1, 0, "f16", 1), ("large", 1, 1, "bf16", 1)])
def test_step_matches_the_definition(layers, W, pad, dtype, shift):
    c = Case(LAYERS[layers], W, pad, dtype, shift)
    for _ in range(2):  # the second one starts from what the first one left
        want = c.expect()
        kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
        torch.cuda.synchronize()
        c.check(*want)
        assert (c.msg.stats_host()["status"] == 0).all()


@pytest.mark.parametrize("check_finite", [0, 1])
def test_blocks_with_inf_or_nan_are_absent(check_finite):
    c = Case([40, 33, 70000], 3, 2, check_finite=check_finite, hard=False)
    c.grads[1, 39] = float("inf")     # the first layer's short last block
    c.grads[1, 40 + 5] = float("nan")
    c.grads[2, 60000] = -float("inf")
    c.grads[0, 73] = 3e38
    c.state[0, 73] = -3e38            # finite inputs, infinite difference
    want = c.expect()
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    torch.cuda.synchronize()
    c.check(*want)
    assert (c.msg.err.cpu().numpy() == np.inf).tolist() == [[False, False, True], [True, True, False], [False, False, True]]
    assert (c.msg.stats_host()["status"] == (kb.KIMAD_ERR_NONFINITE if check_finite else 0)).all()
    assert (c.msg.scales.cpu().numpy() == 255).sum() == 4
    # the receiver's copy follows, and the absent blocks read as zero
    before = torch.full_like(c.state, 7.0)
    est = before.clone()
    kb.kimad_mx4_apply(c.ctx, c.msg, est)
    out = torch.full_like(c.state, 5.0)
    kb.kimad_mx4_read(c.ctx, c.msg, out)
    torch.cuda.synchronize()
    assert torch.equal(est[1, 32:72], before[1, 32:72]) and not torch.equal(est[1, :32], before[1, :32])
    assert not out[1, 32:72].any() and (out[:, c.N:] == 5.0).all()


@pytest.mark.parametrize("layers,W,pad,shift", [("one", 1, 0, 0), ("edges", 3, 5, 1), ("chunks", 2, 0, 3), ("many", 1, 0, 0)])
def test_receiver_follows_the_sender_bit_for_bit(layers, W, pad, shift):
    c = Case(LAYERS[layers], W, pad, shift=shift)
    copy = c.state.clone()
    for _ in range(2):
        kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
        kb.kimad_mx4_apply(c.ctx, c.msg, copy)
    torch.cuda.synchronize()
    assert np.array_equal(bits(copy), bits(c.state))


@pytest.mark.parametrize("W,pad", [(1, 0), (2, 1), (3, 0), (64, 4)])
def test_model_step_is_that_of_aggregate(W, pad):
    layers = [33, 5000, 1, 256]
    c = Case(layers, W, pad, hard=False, seed=W)
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    gen = torch.Generator(device="cuda").manual_seed(3)
    est = torch.randn((W, c.stride), device="cuda", generator=gen)
    c.msg.scales[0, 2] = 255  # a sender's absent block still counts with its old estimator
    x = torch.randn(c.N + 1, device="cuda", generator=gen)[1:]
    weights = [(m + 1) / 70 for m in range(W)]
    est2, x2 = est.clone(), x.clone()
    kb.kimad_mx4_apply(c.ctx, c.msg, est, x, weights, 0.3)
    kb.kimad_mx4_apply(c.ctx, c.msg, est2)
    kb.kimad_aggregate(x2, est2, weights, 0.3)
    torch.cuda.synchronize()
    assert np.array_equal(bits(est), bits(est2)) and np.array_equal(bits(x), bits(x2))


def test_read_gives_the_values_in_both_types():
    c = Case(LAYERS["edges"] + [70001], 2, 3)
    out, _ = c.expect()
    kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
    for dtype in (torch.float32, torch.bfloat16):
        got = torch.full((2, c.stride), 9.0, dtype=dtype, device="cuda")
        kb.kimad_mx4_read(c.ctx, c.msg, got)
        torch.cuda.synchronize()
        for w in range(2):
            assert same(got[w, :c.N].double().cpu().numpy(), out[w][2])
        assert (got[:, c.N:] == 9.0).all()


def test_any_bytes_are_a_message():
    """Received bytes decide values only: scales of 253 and 254 may overflow, nothing else happens."""
    layers = [100, 33000, 7]
    ctx = kb.new_context(layers, 2, [1.0])
    msg = kb.Mx4Message(ctx)
    rng = np.random.default_rng(1)
    codes, scales = rng.integers(0, 256, msg.codes.shape, dtype=np.uint8), rng.integers(0, 256, msg.scales.shape, dtype=np.uint8)
    msg.codes.copy_(torch.from_numpy(codes))
    msg.scales.copy_(torch.from_numpy(scales))
    out = torch.zeros((2, sum(layers)), device="cuda")
    kb.kimad_mx4_read(ctx, msg, out)
    torch.cuda.synchronize()
    c = np.stack((codes & 15, codes >> 4), -1).reshape(2, -1, 32)
    nb = c.shape[1]
    s = scales[:, :nb].astype(np.float64)
    v = np.where(s == 255, 0.0, 1.0)[..., None] * np.where(c & 8, -1.0, 1.0) * _mx4.GRID[c & 7] * np.exp2(s - 127)[..., None]
    with np.errstate(over="ignore"):
        v = v.astype(np.float32)
    at, b = 0, 0
    for n in layers:
        k = -(-n // 32)
        assert np.array_equal(out[:, at:at + n].cpu().numpy(), v[:, b:b + k].reshape(2, -1)[:, :n])
        at, b = at + n, b + k


def test_both_kinds_of_steps_share_a_context():
    """TopK steps around a 4-bit one: what the one leaves in the workspace does not reach the other."""
    wl = workloads.workload(2, 32)
    r = Runner(wl.layer_sizes, wl.n_workers, wl.ratio_grid, wl.D)
    bw = workloads.bandwidth_trace(wl, 3)
    state = torch.zeros((wl.n_workers, wl.N), device="cuda")
    msg = kb.Mx4Message(r.ctx)
    for s in range(3):
        grads = workloads.gradients(wl, s, device="cuda")
        r.compare_step(grads, state, bw[s], wl.t_target, check_inject=False)
        g = grads.cpu().numpy() - state.cpu().numpy()
        launches = kb.kimad_launch_count(r.ctx)
        kb.kimad_mx4_step(r.ctx, grads, state, msg)
        torch.cuda.synchronize()
        assert kb.kimad_launch_count(r.ctx) == launches + 1
        for w in range(wl.n_workers):
            c, sc, *_ = _mx4.message(g[w], wl.layer_sizes)
            assert np.array_equal(msg.codes[w].cpu().numpy(), c) and np.array_equal(msg.scales[w, :len(sc)].cpu().numpy(), sc)


def test_captured_and_on_another_stream():
    c = Case(LAYERS["chunks"], 2, 1, "bf16", hard=False)
    est, x = torch.zeros_like(c.state), torch.zeros(c.N, device="cuda")
    first = c.state.clone()

    def round_():
        kb.kimad_mx4_step(c.ctx, c.grads, c.state, c.msg)
        kb.kimad_mx4_apply(c.ctx, c.msg, est, x, [0.5, 0.5], 0.1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        round_()
        round_()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    want = [t.clone() for t in (c.state, est, x, c.msg.codes, c.msg.err)]
    c.state.copy_(first)
    est.zero_()
    x.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, (c.state, est, x, c.msg.codes, c.msg.err)):
        assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """Three workers more than 2^30 elements apart: the last one starts behind 2^31 elements."""
    layers = [33, 70000, 5]
    N, stride = sum(layers), (1 << 30) + 4099
    ctx = kb.new_context(layers, 3, [1.0], worker_stride=stride)
    msg = kb.Mx4Message(ctx)
    rng = np.random.default_rng(4)
    g = rng.standard_normal((3, N)).astype(np.float32)
    grads = torch.zeros(2 * stride + N, dtype=torch.bfloat16, device="cuda").as_strided((3, N), (stride, 1))
    state = torch.zeros(2 * stride + N, device="cuda").as_strided((3, N), (stride, 1))
    grads.copy_(torch.from_numpy(g))
    kb.kimad_mx4_step(ctx, grads, state, msg)
    torch.cuda.synchronize()
    d = grads.float().cpu().numpy()
    for w in range(3):
        c, sc, v, _, _ = _mx4.message(d[w], layers)
        assert np.array_equal(msg.codes[w].cpu().numpy(), c) and np.array_equal(msg.scales[w, :len(sc)].cpu().numpy(), sc)
        assert np.array_equal(state[w].cpu().numpy().astype(np.float64), v)
    first = state.clone()
    x = torch.zeros(N, device="cuda")
    kb.kimad_mx4_apply(ctx, msg, state, x, [1.0, 1.0, 1.0], 1.0)
    kb.kimad_mx4_read(ctx, msg, grads)
    torch.cuda.synchronize()
    assert torch.equal(state, 2 * first) and torch.equal(grads.float(), first)
    assert torch.equal(x, -(state[0] + state[1] + state[2]))


# ----------------------------------------------------------------------------- operands
def _guarded(n):
    """n bytes on the device between two walls."""
    t = torch.full((n + 1024,), 0xEE, dtype=torch.uint8, device="cuda")
    return t, t[512:512 + n]


@pytest.mark.parametrize("rows,cols,batch,pad,dtype", [
    (1, 1, 1, 0, "f32"), (1, 2048, 1, 0, "bf16"), (31, 33, 1, 1, "f32"), (32, 128, 2, 0, "bf16"), (33, 129, 3, 3, "f16"), (127, 5, 1, 0, "f32"),
    (128, 128, 1, 0, "f32"), (129, 257, 2, 8, "bf16"), (300, 1, 1, 0, "f32"), (1000, 513, 1, 0, "bf16"), (5, 4099, 1, 1, "f32")])
@pytest.mark.parametrize("along", [0, 1])
def test_quantize_and_back(rows, cols, batch, pad, dtype, along):
    rng = np.random.default_rng(rows * 7 + cols)
    v = _mx4.hard_values((batch, rows, cols), rng)
    if dtype == "f16":
        v = np.clip(v, -60000, 60000)
    if batch > 1:
        v[1, 0, 0] = np.inf
        v[1, -1, -1] = np.nan
    room = torch.full((batch, rows, cols + pad), 3.0, dtype=DT[dtype], device="cuda")
    x = room[..., :cols]
    x.copy_(torch.from_numpy(v))
    v = x.float().cpu().numpy()
    lines, length = (cols, rows) if along == 0 else (rows, cols)
    nc, ns = kb.kimad_mx4_operand_bytes(lines, length)
    wc, codes = _guarded(batch * nc)
    ws, scales = _guarded(batch * ns)
    op = kb.Mx4Operand(lines, length, batch, codes=codes, scales=scales)
    kb.kimad_mx4_quantize(x, op, along)
    outs = [torch.full((batch, rows, cols + pad), 3.0, dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16)]
    for o in outs:
        kb.kimad_mx4_dequantize(op, o[..., :cols], along)
    torch.cuda.synchronize()
    for wall in (wc, ws):
        assert (wall[:512] == 0xEE).all() and (wall[-512:] == 0xEE).all()
    codes, scales = codes.cpu().numpy().reshape(batch, lines, -1), scales.cpu().numpy().reshape(batch, -1)
    for n in range(batch):
        m = v[n].T if along == 0 else v[n]
        c, t, values = _mx4.operand(np.ascontiguousarray(m))
        assert np.array_equal(codes[n], c) and np.array_equal(scales[n], t.reshape(-1))
        for o in outs:
            assert same(o[n, :, :cols].double().cpu().numpy(), values.T if along == 0 else values)
    assert (room[..., cols:] == 3.0).all() and all((o[..., cols:] == 3.0).all() for o in outs)


def test_quantize_reads_one_matrix_for_a_whole_batch():
    x = torch.randn((40, 50), device="cuda")
    op = kb.Mx4Operand(50, 40, batch=3)
    kb.kimad_mx4_quantize(x[None].expand(3, 40, 50), op, 0)
    one = kb.Mx4Operand(50, 40)
    kb.kimad_mx4_quantize(x, one, 0)
    torch.cuda.synchronize()
    assert all(torch.equal(op.codes[i], one.codes[0]) and torch.equal(op.scales[i], one.scales[0]) for i in range(3))


def test_empty_matrices():
    for shape, lines, length in [((0, 5), 5, 0), ((5, 0), 0, 5), ((0, 0), 0, 0)]:
        op = kb.Mx4Operand(lines, length)
        x = torch.zeros(shape, device="cuda")
        kb.kimad_mx4_quantize(x, op, 0)
        kb.kimad_mx4_dequantize(op, x, 0)
    torch.cuda.synchronize()


def test_under_the_checked_build():
    """The same tests with the library's index tests and canaries on (a process of its own: the library is chosen when it is loaded)."""
    from paper_2312_08053_b200 import build as kbuild

    if os.environ.get("KIMAD_CHECKED") == "1":
        pytest.skip("this process runs the checked build")
    kbuild.build(checked=True)
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "tests/test_gpu_mx4.py"], cwd=ROOT, env=dict(os.environ, KIMAD_CHECKED="1"),
                         capture_output=True, text=True, timeout=900)
    assert res.returncode == 0 and " passed" in res.stdout, res.stdout[-3000:] + res.stderr[-2000:]
