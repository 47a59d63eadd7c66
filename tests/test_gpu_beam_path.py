"""BeamPath: rotated appends, ragged attention, selection and reordering in one run, held against what 64 bits make of every
hypothesis' own tokens, and the same run with its steps replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb
from tests.beam_harness import END, LAYERS, Toy

pytestmark = pytest.mark.gpu
PROMPTS, BEAMS = [70, 1, 130], 3


def test_a_run_against_every_hypothesis_own_tokens():
    t = Toy(BEAMS, PROMPTS)
    t.start()
    G = len(PROMPTS)
    hist = [p.tolist() for p in t.prompt]
    for layer in range(LAYERS):
        t.check_layer(layer, [g * BEAMS for g in range(G)], hist, [0] * G)
    want = og.beam_select(t.first.double().cpu().numpy(), None, None, 1, BEAMS)
    hyps = [hist[g] for g in range(G) for _ in range(BEAMS)]
    assert t.path.tokens.tolist() == [[tok for _, _, tok in w] for w in want]
    for step in range(70):                                              # past a page's end from 70, 1 and 130 tokens
        tokens, scores, ended = (x.view(-1).cpu().numpy().copy() for x in (t.path.tokens, t.path.scores, t.path.finished))
        hyps = [h + [int(x)] for h, x in zip(hyps, tokens)]
        if step == 3:
            t.path.finished[0, 1] = ended[1] = 1                        # (an end that the toy may not come to by itself)
        t.step()
        assert t.path.status_code() == rb.RTP_OK
        want = og.beam_select(t.last.double().cpu().numpy(), scores, ended, BEAMS, BEAMS, 0)
        parents = [r for w in want for _, r, _ in w]
        assert t.path.parents.view(-1).tolist() == parents and t.path.tokens.view(-1).tolist() == [tok for w in want for _, _, tok in w]
        assert t.path.finished.view(-1).tolist() == [int(ended[r] or tok == END) for w in want for _, r, tok in w]
        hyps = [hyps[r] for r in parents]
        if step % 10 == 4 or step == 69:
            for layer in range(LAYERS):
                back = t.outs[layer], t.lses[layer]
                t.outs[layer], t.lses[layer] = back[0][parents], back[1][parents]   # the rows of the step moved with their sequences
                t.check_layer(layer, range(G * BEAMS), hyps, [len(h) - 1 for h in hyps])
                t.outs[layer], t.lses[layer] = back
                refs = np.zeros(len(t.kv[layer][0]), int)
                table = t.pools[layer].block_table.cpu().numpy()
                np.add.at(refs, table[table >= 0], 1)
                assert (refs == t.pools[layer].page_refs.cpu().numpy()).all()
                assert t.pools[layer].seq_lens.tolist() == [len(h) for h in hyps]


@pytest.mark.parametrize("beams", [1, 4])
def test_replayed_steps(beams):
    """The same bits whether the steps are called or replayed, a warm-up in front or not."""
    runs = []
    for graph in (False, True):
        t = Toy(beams, [63, 5])
        t.start()
        seen = []
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            t.step()
            t.step()
            if graph:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=s):
                    t.step()
            for _ in range(12):
                g.replay() if graph else t.step()
                seen.append([x.clone() for x in (t.path.tokens, t.path.parents, t.path.scores, t.last, t.pools[0].seq_lens)])
        torch.cuda.synchronize()
        assert t.path.status_code() == rb.RTP_OK
        runs.append(seen)
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_full_pool_is_reported():
    t = Toy(2, [64, 64], pages=3)
    t.start()
    assert t.path.status_code() == rb.RTP_OK
    t.step()                                                            # four sequences need a page each, one is left
    assert t.path.status_code() == rb.RTP_ERR_CAPACITY
