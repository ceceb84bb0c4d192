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


@pytest.mark.parametrize("m,n,length", [(300, 200, 64), (128, 128, 8192)])
def test_a_product_without_a_status_of_its_own_is_not_silent(limit, m, n, length):
    """The operands are withheld, by pairs and by parts: the device's status says so until it is reset."""
    a, b, out = ones(m, length), ones(n, length), torch.zeros((m, n), device="cuda")
    kb.kimad_mx4_product_status(reset=True)  # (what tests before this one have left)
    kb.kimad_mx4_product(a, b, out)
    assert kb.kimad_mx4_product_status() == 0 and (out == float(length)).all()
    limit(200000, withhold=True)
    kb.kimad_mx4_product(a, b, out, beta=1.0)
    limit(1 << 31)
    kb.kimad_mx4_product(a, b, out, beta=1.0)  # a call that is right does not cover it up
    assert kb.kimad_mx4_product_status() == kb.KIMAD_ERR_TIMEOUT
    assert kb.kimad_mx4_product_status(reset=True) == kb.KIMAD_ERR_TIMEOUT
    assert kb.kimad_mx4_product_status() == 0
    assert (out == 2.0 * length).all()


def test_a_captured_product_reports_when_it_is_replayed(limit):
    a, out = ones(40, 64), torch.zeros((40, 40), device="cuda")
    kb.kimad_mx4_product_status(reset=True)
    limit(200000, withhold=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kb.kimad_mx4_product(a, a, out)
        with pytest.raises(kb.KimadError) as e:  # nothing could be waited for here; the capture goes on
            kb.kimad_mx4_product_status()
        assert e.value.code == kb.KIMAD_ERR_INVALID_ARG
    limit(1 << 31)
    assert kb.kimad_mx4_product_status() == 0
    for _ in range(2):
        graph.replay()
        assert kb.kimad_mx4_product_status(reset=True) == kb.KIMAD_ERR_TIMEOUT


def test_the_status_can_be_read_on_another_stream(limit):
    a, out, side = ones(40, 64), torch.zeros((40, 40), device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    kb.kimad_mx4_product_status(reset=True)
    limit(200000, withhold=True)
    kb.kimad_mx4_product(a, a, out, stream=side)
    assert kb.kimad_mx4_product_status(reset=True, stream=side) == kb.KIMAD_ERR_TIMEOUT
