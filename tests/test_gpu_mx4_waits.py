"""The bounded waits inside the product: a call that does what it should does not run into them however long its sum, and one that does is not silent."""
import pytest
import torch

from paper_2312_08053_b200 import binding as kb

pytestmark = pytest.mark.gpu


def ones(lines, length):
    """An operand of ones, written as codes and scales: its products are the lengths of the sums, exact in binary32 to 2^24."""
    code_bytes, scale_bytes = kb.kimad_mx4_operand_bytes(lines, length)
    codes, scales = (torch.full((k,), v, dtype=torch.uint8, device="cuda") for k, v in ((code_bytes, 0x22), (scale_bytes, 127)))
    return kb.Mx4Operand(lines, length, codes=codes, scales=scales)


@pytest.fixture
def limit():
    yield kb.kimad_debug_mx4_set_wait_limit
    kb.kimad_debug_mx4_set_wait_limit(1 << 31)


@pytest.mark.parametrize("m,n,length", [(128, 128, 1 << 20), (1280, 1024, 1 << 18)])
def test_the_limit_grows_with_the_sum(limit, m, n, length):
    """By parts and by pairs, 1024 rounds of 256 values a CTA: about 500 000 clocks, with a limit of 131 072 for what does not depend on the sum."""
    a, b = ones(m, length), ones(n, length)
    out, status = torch.zeros((m, n), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    limit(1 << 17)
    kb.kimad_mx4_product(a, b, out, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0 and (out == float(length)).all()
