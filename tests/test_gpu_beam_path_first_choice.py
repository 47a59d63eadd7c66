"""BeamPath: which rows a first choice continues."""
import pytest

from paper_2605_16928_b200 import binding as rb
from tests.beam_harness import Toy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams", [1, 3])
def test_parents_of_a_first_choice_are_the_prompts_rows(beams):
    t = Toy(beams, [7, 70, 1])
    t.start()
    assert t.path.status_code() == rb.RTP_OK
    assert t.path.parents.tolist() == [[g * beams] * beams for g in range(3)]
    table, lens = t.pools[0].block_table.cpu(), t.pools[0].seq_lens.tolist()
    for row, parent in enumerate(t.path.parents.view(-1).tolist()):   # (sequences are numbered like rows)
        assert (table[row] == table[parent]).all() and lens[row] == lens[parent] == [7, 70, 1][row // beams]
