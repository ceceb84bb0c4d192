"""4-bit calls that have to be refused before anything is launched, without a GPU."""
import ctypes as C

import pytest

from paper_2312_08053_b200 import binding as kb
from paper_2312_08053_b200 import build as kbuild

BAD = kb.KIMAD_ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


@pytest.mark.parametrize("err,stats", [(257, 256), (258, 256), (256, 257), (256, 260), (256, 268)])
def test_step_refuses_errors_and_statistics_that_are_not_aligned(err, stats):
    """err is written as f32, stats as records that start with 64-bit words: elsewhere the kernel would fault."""
    L, ctx = kb.load(), kb.kimad_create([40, 7], 2, [1.0])

    def call(e, s):
        return L.kimad_mx4_step(ctx.handle, 256, 0, 512, C.byref(kb.kimad_mx4_message(256, 256, e, s)), None)

    assert call(260, 264) == kb.KIMAD_ERR_WORKSPACE  # everything is right but the workspace, which comes last
    assert call(err, stats) == BAD


@pytest.mark.parametrize("layers", [[40, 33], [33, 41], [33, 64]])
def test_messages_of_contexts_with_other_layers_are_refused(layers):
    """The blocks of [33, 40] are those of these contexts in number, not in place."""
    import torch

    of, to = kb.kimad_create([33, 40], 2, [1.0]), kb.kimad_create(layers, 2, [1.0])
    assert kb.kimad_mx4_message_bytes(of) == kb.kimad_mx4_message_bytes(to)
    msg, t = kb.Mx4Message(of, device="cpu"), torch.zeros((2, sum(layers)))
    for call in (lambda: kb.kimad_mx4_step(to, t, t.clone(), msg), lambda: kb.kimad_mx4_apply(to, msg, t), lambda: kb.kimad_mx4_read(to, msg, t)):
        with pytest.raises(ValueError, match="another context's shape"):
            call()


def test_messages_of_contexts_with_the_same_layers_are_taken():
    """Whatever else the contexts differ in.  (What is refused here is a tensor in host memory.)"""
    import torch

    of, to = kb.kimad_create([33, 40], 2, [1.0]), kb.kimad_create([33, 40], 2, [0.1, 1.0], worker_stride=80, policy=1)
    msg = kb.Mx4Message(of, device="cpu")
    with pytest.raises(ValueError, match="host memory"):
        kb.kimad_mx4_read(to, msg, torch.zeros((2, 80)))


@pytest.mark.parametrize("ld,batch_stride", [(9, 4), (10, 4), (9, 5), (39, 0), (1 << 63, 0), (14, 6), (6, 1), (15, 1 << 63)])
def test_outputs_on_top_of_each_other_are_refused(ld, batch_stride):
    """Three matrices of 7 by 5: behind each other they need batch_stride >= 6 ld + 5, beside each other batch_stride >= 5 and ld >= 2 batch_stride + 5."""
    L, one, zero = kb.load(), C.c_float(1), C.c_float(0)
    assert L.kimad_mx4_dequantize(512, 1024, 256, 0, 7, 5, ld, 3, batch_stride, 1, None) == BAD
    assert L.kimad_mx4_product(256, ld, batch_stride, 7, 5, 40, 3, 512, 1024, 2048, 4096, one, zero, None, None) == BAD
