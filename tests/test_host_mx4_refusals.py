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
