"""rtp_beam_select where a beam's score makes different logits equal: scores[b] + logit in 64 bits decides, equal ones go by (b, t)."""
import numpy as np
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from tests.test_gpu_beam import i32, select

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FLT_MAX = 3.4028234663852886e38


def statement(logits, scores, finished, beams, k, pad=3):
    """Per group the k best (row, token), with their scores."""
    x, picked = logits.double().cpu().numpy(), []
    for g in range(len(x) // beams):
        cands = []
        for row in range(g * beams, (g + 1) * beams):
            base = float(scores[row])
            base = base if base < np.inf else -np.inf              # (NaN and +infinity count as -infinity)
            if finished is not None and finished[row]:
                cands.append((-base, row, pad))
                continue
            top = x[row].max()
            a = base + x[row]
            s = a - (top + np.log(np.exp(x[row] - top).sum())) if np.isfinite(top) else np.full(len(a), -np.inf)
            cands += [(-s[t], row, int(t)) for t in np.argsort(-a, kind="stable")[:k]]
        cands.sort(key=lambda c: (c[0], c[1]))                     # (stable: a beam's tokens stay in their order)
        picked.append([(-s, row, t) for s, row, t in cands[:k]])
    return picked


def check(logits, scores, finished, beams, k, code=rb.RTP_OK):
    parent, token, out, got_code = select(logits, torch.tensor(scores, dtype=torch.float32, device=DEV), None if finished is None else i32(finished), beams, k)
    assert got_code == code
    for g, w in enumerate(statement(logits, np.asarray(scores, np.float32), finished, beams, k)):
        n = len(w)
        assert [(int(p), int(t)) for p, t in zip(parent[g], token[g])] == [(r, t) for _, r, t in w] + [(-1, -1)] * (k - n), g
        for i, (s, _, _) in enumerate(w):                          # a rounding to 32 bits and a normaliser within 2^-18
            assert (out[g, i] == s) if np.isinf(s) else abs(out[g, i] - s) <= 2.0 ** -24 * abs(s) + 2.0 ** -18, (g, i, out[g, i], s)


def rows(n, V, dtype, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + V)
    return (torch.randn((n, V), device=DEV, generator=g) * 3).to(dtype)


def test_ten_logits_of_a_beam_that_is_not_in_use():
    check(torch.arange(10.0, device=DEV)[None], [-np.inf], None, 1, 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V,k", [(10, 7), (700, 64), (9001, 33), (70000, 16)])
@pytest.mark.parametrize("score", [-np.inf, -FLT_MAX, FLT_MAX, -1e30])
def test_all_tokens_are_equal(V, k, score, dtype):
    x = rows(3, V, dtype)
    check(x, [score] * 3, None, 1, k)
    check(x, [score] * 3, None, 3, k)                              # (the first beam has enough of them)


@pytest.mark.parametrize("V", [40, 5000, 50001])
def test_beams_that_are_not_in_use_fill_what_is_missing(V):
    """One beam with three tokens, one that has ended, then those that are not in use."""
    x = rows(8, V, torch.float32)
    x[0], x[4] = -torch.inf, -torch.inf
    x[0, [V - 1, 7, 20]] = torch.tensor([1.0, 2.0, 0.5], device=DEV)
    x[4, :2] = 1.0
    x[6, ::3] = -torch.inf                                         # (ruled out or not: all of them are at -infinity)
    x[2, 5] = -FLT_MAX                                             # an ordinary logit, if a low one
    for none in (-FLT_MAX, -1e30, -np.inf):
        check(x, [-1.0, -2.0, none, -np.inf, 0.0, -np.inf, none, none], [0, 1, 0, 0, 0, 1, 0, 0], 4, min(V - 1, 24))
        check(x, [none] * 8, None, 4, 30)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_scores_that_are_no_numbers_count_as_minus_infinity(bad):
    x = rows(4, 3000, torch.float32)
    check(x, [bad, bad, -np.inf, -1.0], None, 1, 5, rb.RTP_ERR_INVALID)
    check(x, [bad, -np.inf, bad, bad], None, 2, 9, rb.RTP_ERR_INVALID)


@pytest.mark.parametrize("V,k", [(300, 40), (20000, 64), (100000, 5)])
def test_differences_that_a_large_score_swallows(V, k):
    """At -1e9 64 bits hold multiples of 2^-23: logits 2^-20 apart differ, those within 2^-24 of each other do not."""
    g = torch.Generator(device=DEV)
    g.manual_seed(V)
    c = torch.randint(0, 1 << 10, (6, V), device=DEV, generator=g).double()
    j = torch.randint(-7, 8, (6, V), device=DEV, generator=g).double()
    x = (c * 2.0 ** -13 + j * 2.0 ** -27).float()                  # (below 1 / 8: exact in 32 bits)
    x[1] = c[1].float() * 2.0 ** -13 * 0 + (j[1] * 2.0 ** -27).float()   # all of them equal at -1e9
    x[3, : V // 2] = x[3, 0]
    check(x, [-1e9] * 6, None, 1, k)
    check(x, [-1e9, -1.0, -1e9, -1e9, 0.0, -1e9], None, 3, k)


def test_more_equal_ones_in_few_threads_than_a_list_holds():
    """Thousands of different logits that are equal under the score lie in a few threads' hands, in rows that are not cut."""
    V = 20000
    x = rows(600, V, torch.float32) * 2.0 ** -30
    t = torch.arange(V, device=DEV)
    x[:, (t % 1024) < 300] += 1.0 / 16
    x[::2, (t % 2048) >= 1400] += 1.0 / 16
    check(x, [-1e9] * 600, None, 1, 64)      # (a beam a group: beams at -1e9 are nearer to each other than their normalisers are known)

