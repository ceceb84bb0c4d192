"""4-bit messages and operands without a GPU: sizes, the refusals of the C calls (which come before any CUDA call) and of the binding, and the
tests' own reference against values worked out by hand."""
import ctypes as C

import numpy as np
import pytest

from paper_2312_08053_b200 import binding as kb
from paper_2312_08053_b200 import build as kbuild
from tests import _mx4

BAD = kb.KIMAD_ERR_INVALID_ARG


@pytest.fixture(scope="module", autouse=True)
def _built():
    kbuild.build()


def _ctx(layers=(40, 7), W=2, **more):
    return kb.kimad_create(list(layers), W, [1.0], **more)


def test_reference_by_hand():
    block = np.zeros(32, np.float32)
    # the largest magnitude 6.5 has exponent 2: scale 1; ties 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5 go to the even codes 0, 2, 2, 4, 4, 6, 6
    block[:12] = [6.5, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5.0, 0.26, -0.0, 7.9, 5.1]
    code, byte, v = _mx4.quantize(block[None])
    assert byte.tolist() == [127]
    assert code[0, :12].tolist() == [7, 8, 2, 2, 12, 4, 6, 6, 1, 8, 7, 7]
    assert v[0, :12].tolist() == [6, -0.0, 1, 1, -2, 2, 4, 4, 0.5, -0.0, 6, 6]
    code, byte, v = _mx4.quantize(block[None] * np.float32(2.0 ** -140))  # subnormal: the smallest scale
    assert byte.tolist() == [0] and not v.any()
    code, byte, v = _mx4.quantize(np.full((1, 32), np.float32(2.0 ** -126)))
    assert byte.tolist() == [0] and (v == 2.0 ** -126).all() and (code == 4).all()
    code, byte, v = _mx4.quantize(np.full((1, 32), np.float32(3.4e38)))
    assert byte.tolist() == [252] and (v == 6 * 2.0 ** 125).all()
    block[3] = np.inf
    code, byte, v = _mx4.quantize(block[None])
    assert byte.tolist() == [255] and not code.any() and np.isnan(v).all()
    tiles = _mx4.scale_tiles(np.arange(130 * 5, dtype=np.int64).reshape(130, 5).astype(np.uint8))
    assert tiles.shape == (2, 2, 512) and tiles[0, 0, 33 % 32 * 16 + 4 + 2] == (33 * 5 + 2) % 256 and tiles[1, 1, 16] == (129 * 5 + 4) % 256


@pytest.mark.parametrize("layers", [[1], [32], [33, 31, 64], [100000, 5, 1, 1, 1]])
def test_message_bytes(layers):
    blocks = sum(-(-n // 32) for n in layers)
    assert kb.kimad_mx4_message_bytes(_ctx(layers)) == (16 * blocks, -(-blocks // 16) * 16)


@pytest.mark.parametrize("lines,length", [(0, 0), (0, 5), (5, 0), (1, 1), (128, 128), (129, 129), (2048, 33), (1 << 30, 1)])
def test_operand_bytes(lines, length):
    blocks = -(-length // 32)
    want = (lines * blocks * 16, -(-lines // 128) * -(-blocks // 4) * 512)
    assert kb.kimad_mx4_operand_bytes(lines, length) == want


def test_operand_bytes_refuses_what_cannot_be_addressed():
    for a in ((1 << 30) + 1, 5), (5, (1 << 30) + 1):
        with pytest.raises(kb.KimadError) as e:
            kb.kimad_mx4_operand_bytes(*a)
        assert e.value.code == BAD


def _msg(codes=256, scales=256, err=256, stats=256):
    return C.byref(kb.kimad_mx4_message(codes, scales, err, stats))


def test_step_refusals():
    L, ctx = kb.load(), _ctx()
    good = [ctx.handle, 256, 0, 512, _msg(), None]
    assert L.kimad_mx4_step(*good) == kb.KIMAD_ERR_WORKSPACE  # everything else is right
    for i, v in [(0, None), (1, None), (1, 258), (2, 3), (3, None), (3, 514), (4, None), (4, _msg(codes=None)), (4, _msg(codes=264)), (4, _msg(scales=None)),
                 (4, _msg(scales=257)), (4, _msg(err=None)), (4, _msg(stats=None))]:
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_step(*a) == BAD, (i, v)
    assert L.kimad_mx4_step(ctx.handle, 257, 1, 512, _msg(), None) == BAD  # bf16 at an odd byte
    assert L.kimad_mx4_step(ctx.handle, 258, 1, 512, _msg(), None) == kb.KIMAD_ERR_WORKSPACE


def test_apply_and_read_refusals():
    L, ctx, w = kb.load(), _ctx(), (C.c_float * 2)(0.5, 0.5)
    good = [ctx.handle, _msg(err=None, stats=None), 512, 1024, w, C.c_float(1.0), None]
    assert L.kimad_mx4_apply(*good) == kb.KIMAD_ERR_WORKSPACE
    for i, v in [(0, None), (1, None), (1, _msg(codes=260)), (2, None), (2, 513), (3, 1026), (4, None)]:
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_apply(*a) == BAD, (i, v)
    many = _ctx(W=65)
    assert L.kimad_mx4_apply(many.handle, _msg(), 512, 1024, w, C.c_float(1.0), None) == BAD  # more senders than the model step takes
    assert L.kimad_mx4_apply(many.handle, _msg(), 512, None, None, C.c_float(1.0), None) == kb.KIMAD_ERR_WORKSPACE
    good = [ctx.handle, _msg(err=None, stats=None), 512, 0, None]
    assert L.kimad_mx4_read(*good) == kb.KIMAD_ERR_WORKSPACE
    for i, v in [(0, None), (1, None), (1, _msg(scales=None)), (2, None), (2, 514), (3, 2), (3, 7)]:
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_read(*a) == BAD, (i, v)


def test_quantize_and_dequantize_refusals():
    L = kb.load()
    # x, dtype, rows, cols, ld, batch, batch_stride, along, codes, scales, stream
    good = [256, 0, 5, 7, 7, 1, 0, 0, 512, 1024, None]
    for i, v in [(0, None), (0, 258), (1, 3), (2, (1 << 30) + 1), (3, (1 << 30) + 1), (4, 6), (7, 2), (8, None), (8, 520), (9, None), (9, 1032),
                 (5, 1 << 31)]:
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_quantize(*a) == BAD, (i, v)
    for i in (2, 3, 5):  # nothing to do
        a = list(good)
        a[i] = 0
        assert L.kimad_mx4_quantize(*a) == kb.KIMAD_OK
    # codes, scales, x, dtype, rows, cols, ld, batch, batch_stride, along, stream
    good = [512, 1024, 256, 0, 5, 7, 8, 2, 39, 1, None]
    for i, v in [(0, None), (0, 520), (1, None), (2, None), (2, 257), (3, 2), (6, 6), (6, 1 << 62), (8, 38), (9, 2)]:  # (4 * 2^62 is no distance in 64 bits)
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_dequantize(*a) == BAD, (i, v)
    for i in (4, 5, 7):
        a = list(good)
        a[i] = 0
        assert L.kimad_mx4_dequantize(*a) == kb.KIMAD_OK


def test_binding_refuses_shapes_types_and_places():
    import torch

    ctx = _ctx((40, 8), W=2)
    msg = kb.Mx4Message(ctx, device="cpu")
    t = torch.zeros((2, 48))
    with pytest.raises(TypeError):
        kb.kimad_mx4_step(ctx, t.double(), t, msg)
    with pytest.raises(TypeError):
        kb.kimad_mx4_step(ctx, t, t.half(), msg)
    with pytest.raises(ValueError):
        kb.kimad_mx4_step(ctx, t[:, :47], t, msg)
    with pytest.raises(ValueError):
        kb.kimad_mx4_step(ctx, torch.zeros((48, 2)).t(), t, msg)
    with pytest.raises(ValueError):
        kb.kimad_mx4_step(ctx, torch.zeros((2, 64))[:, :48], t, msg)  # another stride than the context's
    with pytest.raises(ValueError):
        kb.kimad_mx4_apply(ctx, kb.Mx4Message(_ctx((40, 8), W=1), device="cpu"), t)
    with pytest.raises(TypeError):
        kb.kimad_mx4_read(ctx, msg, t.half())
    op = kb.Mx4Operand(7, 5, batch=3, device="cpu")
    for x, along in [(torch.zeros(3, 5, 7), 1), (torch.zeros(3, 7, 5), 0), (torch.zeros(2, 5, 7), 0), (torch.zeros(5, 7), 0), (torch.zeros(3, 7, 5).transpose(1, 2), 0),
                     (torch.zeros(3, 5, 7), 2), (torch.zeros(1, 7).expand(3, 5, 7), 0)]:
        with pytest.raises(ValueError):
            kb.kimad_mx4_quantize(x, op, along)
    with pytest.raises(TypeError):
        kb.kimad_mx4_quantize(torch.zeros(3, 5, 7, dtype=torch.int32), op, 0)
    with pytest.raises(TypeError):
        kb.kimad_mx4_dequantize(op, torch.zeros(3, 5, 7).half(), 0)
    with pytest.raises(ValueError):
        kb.Mx4Operand(7, 5, codes=torch.zeros(6, dtype=torch.uint8), scales=torch.zeros(512, dtype=torch.uint8))


def test_binding_refuses_a_workspace_of_another_device():
    import torch

    class Elsewhere:
        def get_device(self):
            return 1

    ctx = _ctx((40, 8), W=2)
    msg = kb.Mx4Message(ctx, device="cpu")
    t, x = torch.zeros((2, 48)), torch.zeros(48)
    ctx._keep = [Elsewhere()]
    for call in (lambda: kb.kimad_mx4_step(ctx, t, t.clone(), msg), lambda: kb.kimad_mx4_apply(ctx, msg, t),
                 lambda: kb.kimad_mx4_apply(ctx, msg, t, x, [0.5, 0.5], 0.1), lambda: kb.kimad_mx4_read(ctx, msg, t)):
        with pytest.raises(ValueError, match="different devices"):
            call()


def test_product_refusals():
    L = kb.load()
    # out, ld, batch_stride, m, n, length, batch, a codes, a scales, b codes, b scales, alpha, beta, status, stream
    good = [256, 7, 0, 5, 7, 40, 1, 512, 1024, 2048, 4096, C.c_float(1), C.c_float(0), None, None]
    for i, v in [(0, None), (0, 258), (1, 6), (3, (1 << 30) + 1), (4, (1 << 30) + 1), (5, (1 << 30) + 1), (6, 2), (7, None), (7, 520), (8, None), (8, 1032), (9, None),
                 (9, 2056), (10, None), (10, 4104), (13, 6)]:
        a = list(good)
        a[i] = v
        assert L.kimad_mx4_product(*a) == BAD, (i, v)
    for i in (3, 4, 6):  # nothing to do
        a = list(good)
        a[i] = 0
        assert L.kimad_mx4_product(*a) == kb.KIMAD_OK
    huge = list(good)
    huge[3], huge[4], huge[1], huge[5] = 1 << 24, 1 << 24, 1 << 24, 1  # 2^34 tiles of outputs
    assert L.kimad_mx4_product(*huge) == BAD


def test_binding_refuses_products_of_what_does_not_fit():
    import torch

    def op(lines, length, batch=1):
        return kb.Mx4Operand(lines, length, batch, device="cpu")

    for a, b, out in [(op(5, 40), op(7, 41), torch.zeros(5, 7)), (op(5, 40, 2), op(7, 40), torch.zeros(2, 5, 7)), (op(5, 40), op(7, 40), torch.zeros(7, 5)),
                      (op(5, 40), op(7, 40), torch.zeros(7, 5).t()), (op(5, 40), op(7, 40), torch.zeros(7).expand(5, 7)), (op(5, 40), op(7, 40), torch.zeros(5, 7))]:
        with pytest.raises(ValueError):  # the last one: not on a CUDA device
            kb.kimad_mx4_product(a, b, out)
    with pytest.raises(TypeError):
        kb.kimad_mx4_product(op(5, 40), op(7, 40), torch.zeros(5, 7, dtype=torch.bfloat16))


def test_wait_limit_is_validated():
    kb.kimad_debug_mx4_set_wait_limit(5, withhold=True)
    kb.kimad_debug_mx4_set_wait_limit(1 << 31)
    with pytest.raises(kb.KimadError) as e:
        kb.kimad_debug_mx4_set_wait_limit((1 << 31) + 1)
    assert e.value.code == BAD
