"""Products into padded rows: what lies between a row's last element and the next row is not the output's."""
import pytest
import torch

from paper_2312_08053_b200 import binding as kb
from tests.test_gpu_mx4_pairs import exact_operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 3, 5, 13, 34, 63, 65, 97, 191, 193, 195, 390])
@pytest.mark.parametrize("batch,m,length,room", [(1, 5, 40, 4), (2, 130, 300, 8), (3, 300, 64, 32), (2, 128, 6144, 4)])
def test_the_padding_stays_as_it_is(batch, m, n, length, room):
    """Rows on 16 bytes (their distance is a multiple of `room` elements) whose last 16 bytes are not all the output's, by pairs and by parts."""
    (a, va), (b, vb) = exact_operand(batch, m, length, n), exact_operand(batch, n, length, n + 1)
    want = (va @ vb.transpose(1, 2)).float()
    ld = -(-(n + 1) // room) * room
    flat = torch.full((batch * m * ld + 64,), 7.0, device="cuda")
    out = flat[:batch * m * ld].view(batch, m, ld)[..., :n]
    assert out.data_ptr() % 16 == 0 and ld > n
    for beta in (0.0, 2.0):
        out.fill_(3.0)
        kb.kimad_mx4_product(a, b, out, beta=beta)
        torch.cuda.synchronize()
        assert torch.equal(out, want + 3.0 * beta)
        out.fill_(7.0)
        assert (flat == 7.0).all()
