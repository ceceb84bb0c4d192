"""Products by pairs of SMs: what either SM of a pair brings (half of the codes, a quarter's scales each) has reached the products that the first one
issues, and sums are taken out before their place is used again.  Operands change from launch to launch and every line differs, so that codes or scales
of another stage, tile or launch would show."""
import pytest
import torch

from paper_2312_08053_b200 import binding as kb

pytestmark = pytest.mark.gpu


def exact_values(shape, seed):
    """Values on the grid with block scales of 1/2, 1 and 2, on the device, and the same in 64 bits.  Products are whole multiples of 1/16 up to 144, so sums
    of up to 7281 of them stay below 2^20: 24 bits, exact in binary32 in whatever order they are added."""
    assert shape[-1] <= 7281
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = -(-shape[-1] // 32)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    v = grid[torch.randint(0, 15, (*shape[:-1], blocks, 32), device="cuda", generator=g)]
    v[..., 0] = 6.0  # the block's scale is known
    v *= torch.tensor([.5, 1., 2.], device="cuda")[torch.randint(0, 3, (*shape[:-1], blocks, 1), device="cuda", generator=g)]
    return v.flatten(-2)[..., :shape[-1]].contiguous()


def exact_operand(batch, lines, length, seed):
    v = exact_values((batch, lines, length), seed)
    op = kb.Mx4Operand(lines, length, batch)
    kb.kimad_mx4_quantize(v, op, 1)
    return op, v.double()


@pytest.mark.parametrize("batch,m,n,length", [
    (1, 2560, 1536, 6400),  # 25 rounds a tile, two tiles and more a pair
    (3, 1100, 900, 257),    # a second round of one block
    (40, 300, 200, 700),    # the second SM has 44 lines of its 128
    (2, 100, 2000, 1000)])  # ... and none
@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_both_halves_of_every_stage_are_those_of_this_launch(batch, m, n, length, beta):
    sets = [(exact_operand(batch, m, length, 2 * i), exact_operand(batch, n, length, 2 * i + 1)) for i in range(3)]
    wants = [(a[1] @ b[1].transpose(1, 2)).float() for a, b in sets]
    outs = [torch.full((batch, m, n), float(i), device="cuda") for i in range(12)]
    torch.cuda.synchronize()
    for i, out in enumerate(outs):  # behind each other, without a pause
        a, b = sets[i % 3]
        kb.kimad_mx4_product(a[0], b[0], out, beta=beta)
    torch.cuda.synchronize()
    for i, out in enumerate(outs):
        assert torch.equal(out, wants[i % 3] + beta * i)
