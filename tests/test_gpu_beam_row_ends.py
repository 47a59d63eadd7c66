"""rtp_beam_select where rows begin and end inside a 16-byte piece: every remainder with every alignment."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_beam import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("whole", [0, 2040, 4096])
def test_every_remainder_and_alignment(whole, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(whole)
    n = 16 // dtype.itemsize
    for rest in range(1, 2 * n + 1):
        V = whole + rest
        for skew in range(n):                      # row r begins r * skew elements behind a boundary
            stride = -(-V // n) * n + n + skew
            x = torch.full((n + 1, stride), torch.nan, device=DEV, dtype=dtype)   # (what lies between the rows is not read)
            x[:, :V] = (torch.randn((n + 1, V), device=DEV, generator=g) * 3).to(dtype)
            x[:, V - 1] = 9                        # the last token of each row is its best, the first one next
            x[:, 0] = 8
            assert check(x[:, :V], None, None, n + 1, min(V, 7)) == rb.RTP_OK, (V, stride)
