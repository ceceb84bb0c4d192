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
