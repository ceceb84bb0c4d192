"""Products whose sum is shared by two or four CTAs, exact to the last bit: alone, beside others, after a failure."""
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from tests.test_gpu_mx4_pairs import exact_operand

pytestmark = pytest.mark.gpu
# two and four CTAs to a tile; the last one's part of the sum whole, cut short, or one round of a single block
SHAPES = [(1, 200, 130, 4500), (1, 128, 128, 6144), (2, 300, 500, 7281), (9, 130, 256, 4097), (1, 129, 1, 5000), (4, 256, 256, 3329), (37, 20, 140, 7200)]


def _case(batch, m, n, length):
    (a, va), (b, vb) = exact_operand(batch, m, length, m + length), exact_operand(batch, n, length, n + length + 1)
    return a, b, (va @ vb.transpose(1, 2)).float()


@pytest.mark.parametrize("batch,m,n,length", SHAPES)
def test_exact_sums(batch, m, n, length):
    a, b, want = _case(batch, m, n, length)
    for beta in (0.0, 1.0):
        out = torch.full((batch, m, n), 2.0, device="cuda")
        kb.kimad_mx4_product(a, b, out, beta=beta)
        assert torch.equal(out, want + 2.0 * beta)


def test_beside_each_other_on_streams_and_from_graphs():
    cases = [_case(*s) for s in SHAPES[:4]] + [_case(2, 2560, 700, 300)]  # the last one by pairs
    streams, outs = [torch.cuda.Stream() for _ in cases], [torch.zeros_like(c[2]) for c in cases]
    kb.kimad_mx4_product_status(reset=True)
    torch.cuda.synchronize()
    for _ in range(10):
        for (a, b, _), out, s in zip(cases, outs, streams):
            kb.kimad_mx4_product(a, b, out, beta=1.0, stream=s)
    torch.cuda.synchronize()
    for i, (c, out) in enumerate(zip(cases, outs)):
        sum_ = torch.zeros_like(out)
        for _ in range(10):
            sum_ += c[2]
        assert torch.equal(out, sum_), i
    graphs = []
    for a, b, want in cases:
        out, g = torch.zeros_like(want), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kb.kimad_mx4_product(a, b, out)
        graphs.append((g, out, want))
    for _ in range(3):
        for (g, _, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for _, out, want in graphs)
    assert kb.kimad_mx4_product_status() == 0


@pytest.mark.parametrize("batch,m,n,length", [(1, 128, 128, 6144), (2, 300, 500, 7281), (1, 600, 500, 700)])
def test_exact_after_a_failure(batch, m, n, length):
    """Operands are withheld (a wait of 0.1 ms runs out); the next call, right behind, is exact."""
    a, b, want = _case(batch, m, n, length)
    out = torch.full_like(want, 3.0)
    kb.kimad_mx4_product_status(reset=True)
    kb.kimad_debug_mx4_set_wait_limit(200000, withhold=True)
    try:
        kb.kimad_mx4_product(a, b, out, beta=1.0)
    finally:
        kb.kimad_debug_mx4_set_wait_limit(1 << 31)
    kb.kimad_mx4_product(a, b, out, beta=1.0)
    assert kb.kimad_mx4_product_status(reset=True) == kb.KIMAD_ERR_TIMEOUT
    assert torch.equal(out, want + 3.0)
