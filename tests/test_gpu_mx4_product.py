"""The product of two operands in 4-bit blocks against the same sums in 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from tests import _mx4

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def operand(m):
    """f32 [batch, lines, length] -> (device operand packed on the host, its values in 64 bits)."""
    parts = [_mx4.operand(x) for x in m]
    codes = torch.from_numpy(np.stack([p[0] for p in parts])).cuda()
    scales = torch.from_numpy(np.stack([p[1] for p in parts])).cuda()
    return kb.Mx4Operand(m.shape[1], m.shape[2], len(m), codes=codes, scales=scales), np.stack([p[2] for p in parts])


def output(batch, m, n, pad=0, gap=0, shift=0, seed=0):
    """A place in a flat vector whose other elements must not change."""
    rng = np.random.default_rng(seed)
    stride = m * (n + pad) + gap
    flat = torch.from_numpy(rng.standard_normal(shift + batch * stride + 64).astype(np.float32)).cuda()
    return flat, flat[shift:shift + batch * stride].view(batch, stride)[:, :m * (n + pad)].view(batch, m, n + pad)[..., :n]


def check_rest(before, flat, out):
    """Everything of `flat` but `out` is as it was."""
    out.copy_(torch.zeros_like(out))
    now = flat.clone()
    flat.copy_(before)
    out.copy_(torch.zeros_like(out))
    assert torch.equal(now, flat)


def exact_matrix(shape, rng):
    """Values on the grid with block scales of 1/2, 1 and 2: sums of up to a thousand products are whole multiples of 1/16 below 2^20, exact in
    binary32 in whatever order they are added."""
    n = -(-shape[-1] // 32)
    v = rng.choice(np.concatenate((_mx4.GRID, -_mx4.GRID)), shape[:-1] + (n, 32))
    v[..., 0] = 6.0  # the block's scale is known
    v = (v * rng.choice([.5, 1., 2.], v.shape[:-1])[..., None]).reshape(shape[:-1] + (-1,))[..., :shape[-1]]
    return np.ascontiguousarray(v, dtype=np.float32)


SHAPES = [(1, 1, 1, 1), (1, 128, 128, 64), (1, 128, 128, 256), (1, 7, 300, 33), (1, 300, 7, 65), (2, 129, 127, 31), (3, 64, 257, 97), (1, 130, 131, 129),
          (1, 256, 384, 1000), (4, 20, 30, 511), (1, 1, 1000, 257), (2, 513, 1, 768), (1, 128, 128, 800),
          # few tiles and a long sum: shared by two and by four CTAs, the last of which may be left with nothing
          (1, 256, 200, 3073), (1, 130, 129, 4097), (2, 70, 60, 4351), (9, 200, 256, 4100), (1, 1, 1, 3329), (36, 128, 128, 4096),
          # outputs on 16 bytes and smaller than a slab; cut tiles of 256 x 192, whole ones, more tiles than pairs of SMs, more rounds than stages
          (3, 5, 8, 100), (1, 40, 36, 70), (2, 300, 12, 65), (2, 300, 200, 2000), (1, 520, 400, 1500),
          (1, 2560, 1536, 64), (40, 130, 200, 300), (80, 20, 30, 511), (1, 2500, 2000, 33), (3, 1300, 1000, 1000), (19, 257, 193, 900), (3, 1300, 1000, 2900), (76, 256, 192, 256)]


@pytest.mark.parametrize("batch,m,n,length", SHAPES)
def test_exact_sums(batch, m, n, length):
    rng = np.random.default_rng(m * 1000 + n + length)
    a, va = operand(exact_matrix((batch, m, length), rng))
    b, vb = operand(exact_matrix((batch, n, length), rng))
    want = np.matmul(va, vb.transpose(0, 2, 1))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for pad, gap, shift in ((0, 0, 0), (3, 1, 1), (4, 8, 4)):
        flat, out = output(batch, m, n, pad, gap, shift)
        before = flat.clone()
        kb.kimad_mx4_product(a, b, out, status=status)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), want)
        assert int(status) == 0
        check_rest(before, flat, out)
        out.copy_(torch.round(torch.randn(out.shape, device="cuda") * 8))
        was = out.cpu().numpy().astype(np.float64)
        kb.kimad_mx4_product(a, b, out, alpha=0.5, beta=-2.0, status=status)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), 0.5 * want - 2.0 * was)


@pytest.mark.parametrize("batch,m,n,length", [(1, 200, 150, 5), (2, 130, 70, 777), (1, 256, 300, 4096), (1, 33, 65, 9000), (1, 2304, 1600, 4500)])
def test_sums_of_any_values(batch, m, n, length):
    """Bound: at most one rounding (by less than a step of the binary32 result, 2^-23 of what has been added up so far in magnitude) per 32 values, and
    one each for alpha, beta."""
    rng = np.random.default_rng(length)
    va, vb = (rng.standard_normal((batch, k, length)).astype(np.float32) * np.exp(rng.standard_normal((batch, k, length))).astype(np.float32) for k in (m, n))
    a, va = operand(va)
    b, vb = operand(vb)
    _, out = output(batch, m, n, 1, 0, 3)
    was = out.cpu().numpy().astype(np.float64)
    kb.kimad_mx4_product(a, b, out, alpha=0.75, beta=0.3)
    size = np.matmul(abs(va), abs(vb).transpose(0, 2, 1))
    want = 0.75 * np.matmul(va, vb.transpose(0, 2, 1)) + np.float64(np.float32(0.3)) * was
    bound = 2.0 ** -23 * ((length / 32 + 2) * 0.75 * size + abs(was))
    assert (abs(out.cpu().numpy() - want) <= bound).all()


def test_scales_far_apart():
    """Blocks of very different sizes: 2^-60 to 2^60 a factor, sums still in binary32's range."""
    rng = np.random.default_rng(5)
    size = np.exp2(rng.integers(-60, 61, (1, 1, 10))).repeat(32, -1)[..., :300].astype(np.float32)
    a, va = operand(rng.standard_normal((1, 140, 300)).astype(np.float32) * size)
    b, vb = operand(rng.standard_normal((1, 150, 300)).astype(np.float32) / size)
    _, out = output(1, 140, 150)
    kb.kimad_mx4_product(a, b, out)
    bound = 2.0 ** -23 * 12 * np.matmul(abs(va), abs(vb).transpose(0, 2, 1))
    assert (abs(out.cpu().numpy() - np.matmul(va, vb.transpose(0, 2, 1))) <= bound).all()


def test_lines_with_inf_or_nan_are_nan():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((1, 130, 100)).astype(np.float32), rng.standard_normal((1, 140, 100)).astype(np.float32)
    x[0, 129, 99], y[0, 5, 0], y[0, 127, 40] = np.inf, np.nan, -np.inf
    a, _ = operand(x)
    b, _ = operand(y)
    _, out = output(1, 130, 140)
    kb.kimad_mx4_product(a, b, out)
    want = np.zeros((130, 140), bool)
    want[129], want[:, 5], want[:, 127] = True, True, True
    assert np.array_equal(np.isnan(out[0].cpu().numpy()), want)


def test_nothing_to_sum_and_nothing_to_write():
    e = kb.Mx4Operand(40, 0, batch=2), kb.Mx4Operand(50, 0, batch=2)
    flat, out = output(2, 40, 50, 2, 3, 1)
    was = out.clone()
    kb.kimad_mx4_product(*e, out, alpha=3.0, beta=-0.5)
    assert torch.equal(out, was * -0.5)
    out.fill_(float("nan"))
    kb.kimad_mx4_product(*e, out, beta=0.0)  # not read
    assert not out.any()
    for m, n, batch in ((0, 5, 1), (5, 0, 1), (5, 5, 0)):
        a, b = kb.Mx4Operand(m, 64, batch=batch), kb.Mx4Operand(n, 64, batch=batch)
        kb.kimad_mx4_product(a, b, torch.zeros((batch, m, n), device="cuda"))
    torch.cuda.synchronize()


def test_beta_zero_does_not_read_the_output():
    rng = np.random.default_rng(3)
    a, va = operand(exact_matrix((1, 50, 64), rng))
    out = torch.full((50, 50), float("nan"), device="cuda")
    kb.kimad_mx4_product(a, a, out)
    assert np.array_equal(out.cpu().numpy().astype(np.float64), va[0] @ va[0].T)  # (and an operand may be both factors)


def test_same_bits_every_time_captured_and_on_another_stream():
    g = torch.Generator(device="cuda").manual_seed(4)
    x, y = (torch.randn((2, 3000, k), device="cuda", generator=g) for k in (260, 200))
    a, b = kb.Mx4Operand(260, 3000, batch=2), kb.Mx4Operand(200, 3000, batch=2)
    out = [torch.zeros((2, 260, 200), device="cuda") for _ in range(3)]

    def pass_(o):
        kb.kimad_mx4_quantize(x, a, 0)
        kb.kimad_mx4_quantize(y, b, 0)
        kb.kimad_mx4_product(a, b, o, alpha=0.5, beta=1.0)

    pass_(out[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        pass_(out[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pass_(out[2])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


def test_a_round_with_factors_and_messages():
    """As they are used together: every worker sends a linear layer's gradient as its two factors (the product goes straight into the layer's place of the
    receiver's flat gradients), compresses the whole vector with 4-bit blocks, and the receiver follows and takes the model step."""
    T, d_in, d_out, W = 70, 129, 66, 2
    layers = [5, d_in * d_out, 33]
    N = sum(layers)
    g = torch.Generator(device="cuda").manual_seed(6)
    x, dy = torch.randn((W, T, d_in), device="cuda", generator=g).bfloat16(), torch.randn((W, T, d_out), device="cuda", generator=g).bfloat16()
    a, b = kb.Mx4Operand(d_in, T, batch=W), kb.Mx4Operand(d_out, T, batch=W)
    kb.kimad_mx4_quantize(x, a, 0)
    kb.kimad_mx4_quantize(dy, b, 0)
    grads = torch.randn((W, N), device="cuda", generator=g)
    kb.kimad_mx4_product(a, b, grads[:, 5:5 + d_in * d_out].unflatten(1, (d_in, d_out)), alpha=1.0 / T, beta=0.0)
    va = [_mx4.operand(np.ascontiguousarray(t.float().cpu().numpy().T))[2] for t in x]
    vb = [_mx4.operand(np.ascontiguousarray(t.float().cpu().numpy().T))[2] for t in dy]
    for w in range(W):
        got = grads[w, 5:5 + d_in * d_out].view(d_in, d_out).cpu().numpy()
        bound = 2.0 ** -23 * (T / 32 + 3) / T * (abs(va[w]) @ abs(vb[w]).T)
        assert (abs(got - va[w] @ vb[w].T / T) <= bound).all()
    ctx = kb.new_context(layers, W, [1.0])
    msg = kb.Mx4Message(ctx)
    state, est, model = torch.zeros((W, N), device="cuda"), torch.zeros((W, N), device="cuda"), torch.zeros(N, device="cuda")
    left = []
    for _ in range(4):
        kb.kimad_mx4_step(ctx, grads, state, msg)
        kb.kimad_mx4_apply(ctx, msg, est, model, [0.5, 0.5], 1.0)
        left.append(msg.stats_host()["total_err"].sum())
    assert torch.equal(est, state)
    # every pass leaves at most a quarter of a value (cut at 6 of up to 8 scales) or half a unit of the block's scale: what is left shrinks
    assert all(q < p for p, q in zip(left, left[1:]))


def test_offsets_beyond_32_bits():
    """Matrices of a batch more than 2^31 elements apart, on 16 bytes (by TMA) and not."""
    rng = np.random.default_rng(8)
    a, va = operand(exact_matrix((3, 130, 70), rng))
    b, vb = operand(exact_matrix((3, 200, 70), rng))
    want = np.matmul(va, vb.transpose(0, 2, 1))
    stride = (1 << 30) + 4096
    flat = torch.zeros(2 * stride + 130 * 204 + 64, device="cuda")
    for shift, ld in ((0, 200), (1, 203)):
        out = flat.as_strided((3, 130, 200), (stride, ld, 1), shift)
        out.copy_(torch.ones((), device="cuda").expand(3, 130, 200))
        kb.kimad_mx4_product(a, b, out, alpha=1.0, beta=2.0)
        assert np.array_equal(out.cpu().numpy().astype(np.float64), want + 2.0)
    x = flat.as_strided((3, 70, 130), (stride, 131, 1), 5)
    x.copy_(torch.randn((3, 70, 130), device="cuda"))
    op, back = kb.Mx4Operand(130, 70, batch=3), torch.zeros((3, 70, 130), device="cuda")
    kb.kimad_mx4_quantize(x, op, 0)
    kb.kimad_mx4_dequantize(op, back, 0)
    values = np.stack([_mx4.operand(np.ascontiguousarray(m.cpu().numpy().T))[2].T for m in x])
    assert np.array_equal(back.cpu().numpy().astype(np.float64), values)
    kb.kimad_mx4_dequantize(op, x, 0)
    assert torch.equal(x, back)


def test_two_at_once_on_streams_given_by_argument():
    """Products by pairs and by parts beside each other, and each replayed from a graph of its own."""
    rng = np.random.default_rng(9)
    work = []
    for m, n, length in ((700, 500, 300), (200, 130, 4500), (40, 36, 64)):
        a, va = operand(exact_matrix((1, m, length), rng))
        b, vb = operand(exact_matrix((1, n, length), rng))
        work.append((a, b, va[0] @ vb[0].T if length <= 1100 else None, [torch.zeros((m, n), device="cuda") for _ in range(3)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for a, b, _, out, s in work:
        kb.kimad_mx4_product(a, b, out[0])
    torch.cuda.synchronize()
    for _ in range(20):
        for a, b, _, out, s in work:
            kb.kimad_mx4_product(a, b, out[1], stream=s)
    torch.cuda.synchronize()
    graphs = []
    for a, b, _, out, s in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kb.kimad_mx4_product(a, b, out[2])
        graphs.append(g)
    for _ in range(5):
        for g, w in zip(graphs, work):
            with torch.cuda.stream(w[4]):
                g.replay()
    torch.cuda.synchronize()
    for _, _, want, out, _ in work:
        assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
        assert want is None or np.array_equal(out[0].cpu().numpy().astype(np.float64), want)


def test_first_calls_of_a_process_can_be_captured():
    code = """
import torch
from paper_2312_08053_b200 import binding as kb
x = torch.randn((300, 200), device="cuda")
a, b = kb.Mx4Operand(200, 300), kb.Mx4Operand(300, 200)
c, d = torch.zeros((200, 200), device="cuda"), torch.zeros((300, 300), device="cuda")
y = torch.zeros_like(x)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
def calls():
    kb.kimad_mx4_quantize(x, a, 0)
    kb.kimad_mx4_quantize(x, b, 1)
    kb.kimad_mx4_product(a, a, c)
    kb.kimad_mx4_product(b, b, d)
    kb.kimad_mx4_dequantize(b, y, 1)
with torch.cuda.graph(g):
    calls()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (c, d, y)]
calls()
torch.cuda.synchronize()
assert all(torch.equal(p, q) and p.any() for p, q in zip(got, (c, d, y)))
print("captured")
"""
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "captured" in res.stdout, res.stdout[-2000:] + res.stderr[-2000:]


@pytest.mark.parametrize("m,n,length", [(600, 500, 700), (128, 128, 8192)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(m, n, length):
    """By pairs and by parts: the operands are not brought, so every wait for them ends at its limit (0.1 ms).  Nothing is written, and the GPU goes on."""
    rng = np.random.default_rng(11)
    a, va = operand(exact_matrix((1, m, length), rng))
    b, vb = operand(exact_matrix((1, n, length), rng))
    want = torch.from_numpy((va[0] @ vb[0].T).astype(np.float32)).cuda()
    for beta in (0.0, 1.0):
        out, status = torch.full((m, n), 3.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        kb.kimad_debug_mx4_set_wait_limit(200000, withhold=True)
        try:
            kb.kimad_mx4_product(a, b, out, beta=beta, status=status)
            torch.cuda.synchronize()
        finally:
            kb.kimad_debug_mx4_set_wait_limit(1 << 31)
        assert int(status) == kb.KIMAD_ERR_TIMEOUT and (out == 3.0).all()
    status.zero_()
    kb.kimad_mx4_product(a, b, out, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and (torch.equal(out, want) if length <= 3000 else torch.allclose(out, want, rtol=1e-5, atol=1e-2 * length))
