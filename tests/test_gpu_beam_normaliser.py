"""rtp_beam_select: the normaliser of rows so many that each CTA would have a whole one, however long."""
import numpy as np
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_beam import select

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(x, distinct):
    """Rows r, r + distinct, .. are equal."""
    parent, token, out, code = select(x, None, None, 1, 1)
    assert code == rb.RTP_OK
    for r in range(distinct):
        y = x[r].double()
        want = float(y.max() - torch.logsumexp(y, 0))
        # the normaliser is right to 2^-16, and the score is rounded to 32 bits
        assert (np.abs(out[r::distinct, 0].astype(np.float64) - want) <= 2.0 ** -16 + 2.0 ** -24 * abs(want)).all(), (r, out[r, 0] - want)
        assert (out[r::distinct] == out[r, 0]).all() and token[r, 0] == int(y.argmax())


def test_terms_that_all_round_alike():
    """Sums of 16 exp(-c) of which 2047, added one after the other in 32 bits, lose 2^-15 of their sum (c chosen for that)."""
    V, c = 1 << 23, np.float32(0.1007995456457138)
    e = np.float32(np.exp2(np.float64(np.float32(-c * np.float32(1.4426950408889634)))))
    w, total = np.float32(16) * e, np.float32(16)
    for _ in range(2047):
        total = np.float32(total + w)
    assert abs(float(total) / (16 + 2047 * 16 * float(e)) - 1) > 2.0 ** -15.5
    x = torch.full((600, V), -float(c), device=DEV)
    x[:, :4096] = 0.0                              # the maximum of every thread
    check(x, 1)


@pytest.mark.parametrize("V,dtype", [(50000, torch.float32), (131072, torch.float32), (131073, torch.bfloat16), (200001, torch.float16), (1 << 21, torch.bfloat16)])
def test_rows_that_rise_fall_and_lie_flat(V, dtype):
    x = torch.empty((600, V), device=DEV, dtype=dtype)
    x[0::4] = torch.linspace(-40, 0, V, device=DEV).to(dtype)      # every piece has a new maximum
    x[1::4] = torch.linspace(0, -40, V, device=DEV).to(dtype)
    x[2::4] = -0.1
    x[3::4] = torch.linspace(-0.5, 0, V, device=DEV).to(dtype)
    check(x, 4)


def test_rows_of_millions_of_tokens_and_tens_of_thousands_of_lists():
    V, W, k = (1 << 25) - 1, 64, 5
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn((W, V), device=DEV, generator=g)
    parent, token, out, code = select(x, None, None, W, k)
    assert code == rb.RTP_OK
    best = []
    for b in range(W):
        v, t = torch.topk(x[b], k)
        norm = float(torch.logsumexp(x[b].double(), 0))
        best += [(norm - float(s), b, int(i)) for s, i in zip(v, t)]
    best.sort()
    best = best[:k]
    assert min(b[0] - a[0] for a, b in zip(best, best[1:])) > 2.0 ** -14     # (apart enough for two normalisers' errors)
    assert [(int(p), int(t)) for p, t in zip(parent[0], token[0])] == [(b, t) for _, b, t in best]
    assert all(abs(out[0, i] + s) <= 2.0 ** -16 + 2.0 ** -24 * s for i, (s, _, _) in enumerate(best))
