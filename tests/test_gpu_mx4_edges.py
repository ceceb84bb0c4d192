"""Ends of what the 4-bit calls' documentation allows."""
import threading

import pytest
import torch

from paper_2312_08053_b200 import binding as kb

pytestmark = pytest.mark.gpu


def test_first_calls_of_a_thread():
    """A thread that has made no CUDA call yet: the tensor maps are made before the first launch."""
    x = torch.randn((300, 200), device="cuda")
    a, want = kb.Mx4Operand(200, 300), torch.zeros((200, 200), device="cuda")
    kb.kimad_mx4_quantize(x, a, 0)
    kb.kimad_mx4_product(a, a, want)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    failures = []

    def call():
        try:
            kb.kimad_mx4_product(a, a, out)
        except Exception as e:
            failures.append(e)

    t = threading.Thread(target=call)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failures and torch.equal(out, want) and want.any()


@pytest.mark.parametrize("alpha", [float("inf"), float("nan"), -float("inf"), -2.0, 3.0])
@pytest.mark.parametrize("beta", [0.0, 1.0, -0.5])
def test_nothing_to_sum_leaves_beta_times_the_output_whatever_alpha(alpha, beta):
    a, b = kb.Mx4Operand(40, 0, batch=2), kb.Mx4Operand(50, 0, batch=2)
    was = torch.randn((2, 40, 50), device="cuda")
    was[0, 0, :2] = torch.tensor([0.0, -0.0])
    out = was.clone() if beta else torch.full_like(was, float("nan"))
    kb.kimad_mx4_product(a, b, out, alpha=alpha, beta=beta)
    want = was * beta if beta else torch.zeros_like(was)
    assert torch.equal(out.view(torch.int32), want.view(torch.int32))  # bit for bit, zeros' signs too
