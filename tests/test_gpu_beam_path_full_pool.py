"""BeamPath on a pool that is full: nothing advances, and the step can be made again when there is room."""
import pytest
import torch

from paper_2605_16928_b200 import binding as rb
from tests.beam_harness import DEV, LAYERS, VOCAB, Toy

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_a_step_that_found_no_room_is_made_again():
    t = Toy(2, [64, 64], pages=5)                  # two pages of prompts; the next token needs four
    t.start()
    hist = t.prompt[0].tolist()
    for _ in range(2):
        t.path.advance()
        assert t.path.status_code() == rb.RTP_ERR_CAPACITY
        assert all(p.seq_lens.tolist() == [64] * 4 for p in t.pools)
    for p in t.pools:
        p.free(i32([2, 3]))                        # the second prompt is given up (its hypotheses begin anew, at position 0)
    t.path.advance()
    assert t.path.status_code() == rb.RTP_OK
    assert all(p.seq_lens.tolist() == [65, 65, 1, 1] for p in t.pools)
    t.attend(t.path.tokens.view(-1).long())
    assert t.path.status_code() == rb.RTP_OK
    tokens = t.path.tokens.view(-1).tolist()
    for layer in range(LAYERS):
        t.check_layer(layer, range(4), [hist + tokens[:1], hist + tokens[1:2], tokens[2:3], tokens[3:]], [64, 64, 0, 0])


def test_one_full_pool_of_several_holds_all_of_them():
    t = Toy(2, [64])
    t.start()
    last = t.pools[-1]
    free = (last.page_refs == 0).nonzero().view(-1)
    last.page_refs[free] = 7                       # (somebody else's)
    t.path.advance()
    assert t.path.status_code() == rb.RTP_ERR_CAPACITY
    assert all(p.seq_lens.tolist() == [64, 64] for p in t.pools)
    last.page_refs[free] = 0
    t.path.advance()
    assert t.path.status_code() == rb.RTP_OK
    assert all(p.seq_lens.tolist() == [65, 65] for p in t.pools)
    t.attend(t.path.tokens.view(-1).long())
    hist = t.prompt[0].tolist()
    for layer in range(LAYERS):
        t.check_layer(layer, range(2), [hist + [x] for x in t.path.tokens.view(-1).tolist()], [64, 64])


def test_prompts_that_find_no_room():
    t = Toy(2, [200, 10], pages=3)
    t.path.prompts([200, 10])
    assert t.path.status_code() == rb.RTP_ERR_CAPACITY
    assert all(p.seq_lens.tolist() == [0] * 4 for p in t.pools)
    t.prompt = [torch.randint(6, VOCAB, (n,), device=DEV) for n in (100, 10)]
    t.start()
    assert t.path.status_code() == rb.RTP_OK
    for layer in range(LAYERS):
        t.check_layer(layer, [0, 2], [p.tolist() for p in t.prompt], [0, 0])
