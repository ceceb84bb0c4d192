"""Batches of matrices that lie beside each other, row by row: [rows][batch][cols] storage, a row of every matrix before the next row of the first."""
import numpy as np
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from tests import _mx4
from tests.test_gpu_mx4_pairs import exact_operand

pytestmark = pytest.mark.gpu


def interleaved(rows, batch, cols, pad, gap, shift, dtype=torch.float32):
    """A flat vector of 7s and the matrices [batch][rows][cols] in it: `pad` elements between matrices, `gap` between rows."""
    stride = cols + pad
    ld = batch * stride + gap
    flat = torch.full((shift + rows * ld + 64,), 7.0, dtype=dtype, device="cuda")
    return flat, flat.as_strided((batch, rows, cols), (stride, ld, 1), shift)


def rest(flat, out):
    """The elements of the vector that are not the matrices', after these have been set to 7."""
    out.fill_(7.0)
    return flat


@pytest.mark.parametrize("rows,cols,batch,pad,gap,shift", [(5, 7, 2, 0, 0, 0), (130, 200, 3, 0, 0, 0), (130, 201, 3, 2, 5, 1), (256, 128, 2, 0, 0, 0), (1, 40, 3, 0, 0, 0), (40, 1, 3, 0, 0, 0)])
@pytest.mark.parametrize("along", [0, 1])
def test_quantised_from_and_read_back_into(rows, cols, batch, pad, gap, shift, along):
    v = _mx4.hard_values((batch, rows, cols), np.random.default_rng(rows + cols))
    _, x = interleaved(rows, batch, cols, pad, gap, shift)
    x.copy_(torch.from_numpy(v))
    lines, length = (cols, rows) if along == 0 else (rows, cols)
    op = kb.Mx4Operand(lines, length, batch)
    kb.kimad_mx4_quantize(x, op, along)
    want = np.stack([_mx4.operand(np.ascontiguousarray(m.T if along == 0 else m))[2] for m in v])
    want = want.transpose(0, 2, 1) if along == 0 else want
    for dtype in (torch.float32, torch.bfloat16):
        flat, back = interleaved(rows, batch, cols, pad, gap, shift, dtype)
        kb.kimad_mx4_dequantize(op, back, along)
        torch.cuda.synchronize()
        assert np.array_equal(back.double().cpu().numpy(), want)
        assert (rest(flat, back) == 7.0).all()


@pytest.mark.parametrize("m,n,batch,length", [(130, 200, 3, 70), (300, 204, 2, 257), (128, 128, 2, 6144), (5, 1, 3, 40)])
@pytest.mark.parametrize("pad,gap,shift", [(0, 0, 0), (4, 8, 4), (1, 3, 5)])
def test_products_into(m, n, batch, length, pad, gap, shift):
    (a, va), (b, vb) = exact_operand(batch, m, length, m), exact_operand(batch, n, length, n)
    want = (va @ vb.transpose(1, 2)).float()
    flat, out = interleaved(m, batch, n, pad, gap, shift)
    for beta in (0.0, 2.0):
        out.fill_(3.0)
        kb.kimad_mx4_product(a, b, out, beta=beta)
        torch.cuda.synchronize()
        assert torch.equal(out, want + 3.0 * beta)
    assert (rest(flat, out) == 7.0).all()
