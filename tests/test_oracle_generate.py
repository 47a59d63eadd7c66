"""Pins of the generation oracle: closed forms and torch's own functions."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as og


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rd", [16, 96, 128])
def test_rotation_keeps_lengths_and_depends_on_differences(rd, interleaved):
    rng = np.random.default_rng(rd)
    q, k = rng.standard_normal((2, 4, 1, 128))
    f = 10000.0 ** (-np.arange(rd // 2) * 2 / rd)
    pos = np.array([0, 1, 77, 100003])
    a, mag = og.rotate(q, pos, f, rd, interleaved)
    assert np.allclose(a[0], q[0]) and np.array_equal(a[..., rd:], q[..., rd:]) and (mag[..., rd:] == 0).all() and (mag[..., :rd] > 0).all()
    assert np.allclose((a ** 2).sum(-1), (q ** 2).sum(-1))
    b, _ = og.rotate(k, pos, f, rd, interleaved)
    c, _ = og.rotate(q, pos + 5000, f, rd, interleaved)
    d, _ = og.rotate(k, pos + 5000, f, rd, interleaved)
    assert np.allclose((a * b).sum(-1), (c * d).sum(-1), atol=1e-9)


def test_rotation_by_a_quarter_turn():
    x = np.zeros((1, 1, 128))
    x[0, 0, 0], x[0, 0, 8] = 3.0, 4.0
    f = np.full(8, np.pi / 2)
    assert np.allclose(og.rotate(x, [1], f, 16)[0][0, 0, [0, 8]], [-4, 3])
    assert np.allclose(og.rotate(x, [1], f, 16, True, 2.0)[0][0, 0, [0, 1, 8, 9]], [0, 6, 0, 8])


def test_attention_is_torchs():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 9, 128))
    o, lse, _ = og.attend(q, k, v, range(9), 0.3)
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)), is_causal=True, scale=0.3)[0]
    assert np.allclose(o, ref.numpy())
    o, lse, _ = og.attend(q, k, v, range(9), 0.3, window=2, n_sink=1)
    mask = np.array([[n <= m and (n < 1 or n > m - 2) for n in range(9)] for m in range(9)])
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)), attn_mask=torch.from_numpy(mask), scale=0.3)[0]
    assert np.allclose(o, ref.numpy())
    o, lse, _ = og.attend(q[:1], k[:0], v[:0], [4], 0.3)
    assert (o == 0).all() and lse[0] == -np.inf


def test_beam_select_is_brute_force():
    rng = np.random.default_rng(2)
    x = np.round(rng.standard_normal((6, 11)) * 2) / 2          # many equal ones
    s = np.array([0, -1, -0.5, 0, -np.inf, -2.0])
    got = og.beam_select(x, s, None, 3, 7)
    ls = torch.log_softmax(torch.from_numpy(x), -1).numpy() + s[:, None]
    for g in range(2):
        every = sorted((-ls[r, t], r, t) for r in range(3 * g, 3 * g + 3) for t in range(11))[:7]
        assert [(r, t) for _, r, t in got[g]] == [(r, t) for _, r, t in every]
    ended = og.beam_select(x, s, [1, 1, 1, 0, 0, 0], 3, 7, pad_token=9)
    assert [(r, t) for _, r, t in ended[0]] == [(0, 9), (2, 9), (1, 9)]
    none = og.beam_select(np.full((1, 4), -np.inf), None, None, 1, 3)
    assert [(r, t) for _, r, t in none[0]] == [(0, 0), (0, 1), (0, 2)] and none[0][0][0] == -np.inf


def test_reorder_permutes_and_counts():
    table = np.array([[0, 1, 4], [0, 2, -1], [0, 3, -1], [5, -1, -1]])
    refs = np.array([3, 1, 1, 1, 1, 1, 0])
    t, lens, r, bad = og.reorder(table, [150, 100, 101, 3], refs, [1, 0, 0], [0, 1, 2])
    assert not bad and (t == [[0, 2, -1], [0, 1, 4], [0, 1, 4], [5, -1, -1]]).all() and (lens == [100, 150, 150, 3]).all()
    assert (r == [3, 2, 1, 0, 2, 1, 0]).all()
    t, lens, r, bad = og.reorder(table, [150, 100, 101, 3], refs, [3, 0, 9], [1, 1, 0])
    assert bad and (t[1] == [5, -1, -1]).all() and (t[0] == table[0]).all() and r[5] == 2
