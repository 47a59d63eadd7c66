"""rtp_beam_select: sums of a large score and logits that are one last place apart, in different slices of a row."""
import pytest
import torch

from tests.test_gpu_beam_ties import DEV, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [12774, 60000])
def test_sums_that_are_one_last_place_apart(V):
    """At -1e9 the sums are multiples of 2^-23; a normaliser half a place off rounds two of them to one."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    x = (torch.randint(0, 40, (64, V), device=DEV, generator=g) * 2.0 ** -23).float()
    x += torch.arange(64, device=DEV)[:, None] * 2.0 ** -28        # (rounded away beside -1e9, or up)
    x[:, 7::1000] += torch.rand((64, len(x[0, 7::1000])), device=DEV, generator=g) * 2.0 ** -20
    check(x, [-1e9] * 64, None, 1, 26)
    check(x.half(), [-1e9] * 64, None, 1, 26)
