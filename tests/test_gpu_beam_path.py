"""BeamPath: rotated appends, ragged attention, selection and reordering in one run, held against what 64 bits make of every
hypothesis' own tokens, and the same run with its steps replayed from a graph."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as og
from paper_2605_16928_b200 import binding as rb
from paper_2605_16928_b200 import pipeline

pytestmark = pytest.mark.gpu
DEV, VOCAB, LAYERS, N_KV, GROUP = "cuda:0", 700, 2, 2, 2
N_Q, WINDOW, SINKS, LOCAL = N_KV * GROUP, 40, 4, 1
PROMPTS, BEAMS, END = [70, 1, 130], 3, 5


class Toy:
    """A model of two layers whose rows depend on the token alone, and whose logits are a fixed projection of the attention."""

    def __init__(self, beams, prompts, pages=None):
        g = torch.Generator(device=DEV)
        g.manual_seed(11)
        self.rows = [torch.randn((VOCAB, N_Q + 2 * N_KV, 128), device=DEV, generator=g).bfloat16() for _ in range(LAYERS)]
        self.head = torch.randn((LAYERS * N_Q * 128, VOCAB), device=DEV, generator=g) * 0.2
        self.prompt = [torch.randint(6, VOCAB, (n,), device=DEV, generator=g) for n in prompts]
        self.freqs = 10000.0 ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64)
        B, cols = len(prompts) * beams, max(prompts) // 64 + 2
        n = pages or B * cols
        self.pools, self.kv = [], []
        for _ in range(LAYERS):
            pool = pipeline.PagePool(rb.Params(N_Q, N_KV, [], [], [], [LOCAL], n_sink=SINKS, window=WINDOW), n, B, cols)
            self.kv.append([torch.full((n, N_KV, 64, 128), torch.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)])
            pool.cache_of(*self.kv[-1])
            self.pools.append(pool)
        self.path = pipeline.BeamPath(self.pools, rb.Rope(self.freqs), len(prompts), beams, VOCAB, sum(prompts), pad_token=0, end_token=END)

    def attend(self, tokens):
        self.outs, self.lses = [], []
        for layer in range(LAYERS):
            x = self.rows[layer][tokens]
            lse = torch.empty((len(x), N_Q), device=DEV)
            self.outs.append(self.path.attend(layer, x[:, :N_Q], x[:, N_Q:N_Q + N_KV], x[:, N_Q + N_KV:], lse=lse))
            self.lses.append(lse)
        return self.outs

    def logits(self, rows=None):
        return torch.cat([(o if rows is None else o[rows]).flatten(1) for o in self.outs], 1).float() @ self.head

    def start(self):
        self.path.prompts([len(p) for p in self.prompt])
        self.attend(torch.cat(self.prompt))
        last = torch.cumsum(torch.tensor([len(p) for p in self.prompt], device=DEV), 0) - 1
        self.first = self.logits(last)
        self.path.begin(self.first)

    def step(self):
        self.path.advance()
        self.attend(self.path.tokens.view(-1).long())
        self.last = self.logits()
        self.path.choose(self.last)

    def check_layer(self, layer, seqs, tokens, pos0):
        """Row i of the last call: the sequence seqs[i], whose tokens are tokens[i], from its position pos0[i] on."""
        table, at = self.pools[layer].block_table.cpu().numpy(), 0
        out, lse = self.outs[layer].float().cpu().numpy(), self.lses[layer].cpu().numpy()
        x = self.rows[layer]
        for s, toks, p0 in zip(seqs, tokens, pos0):
            n, ids = len(toks), torch.tensor(toks, device=DEV)
            pages = torch.tensor(table[s, :-(-n // 64)].astype(np.int64), device=DEV)
            k, v = (a[pages].transpose(1, 2).reshape(-1, N_KV, 128)[:n] for a in self.kv[layer])
            # every cached row is its token's, rotated by its position: one rounding to bf16 on top of 32-bit arithmetic (below 2^-21 of |a| + |b|)
            exact, mag = og.rotate(x[ids, N_Q:N_Q + N_KV].float().cpu().numpy(), np.arange(n), self.freqs.cpu().numpy())
            assert (np.abs(k.float().cpu().numpy() - exact) <= 2.0 ** -8 * np.abs(exact) + mag * 2.0 ** -21 + 1e-38).all()
            assert torch.equal(v, x[ids, N_Q + N_KV:])
            pos = np.arange(p0, n)
            q, qm = og.rotate(x[ids[p0:], :N_Q].float().cpu().numpy(), pos, self.freqs.cpu().numpy())
            kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
            for h in range(N_Q):
                o, l, m = og.attend(q[:, h], kf[:, h // GROUP], vf[:, h // GROUP], pos, 128 ** -0.5, WINDOW if h // GROUP == LOCAL else 0, SINKS)
                # the query is rounded to bf16 first (2^-8 of each element, so 2^-8 |q| |k| / sqrt(128) of a logit at most), then as for the
                # attention alone: 130 x 2^-24 of it for the sums, P and the output 2^-8 each, exponents of two 2^-20
                norm = np.linalg.norm(q[:, h], axis=-1) * np.linalg.norm(kf[:, h // GROUP], axis=-1).max() * 128 ** -0.5
                dz = norm * (2.0 ** -8 + 2.0 ** -21 * 2 + 130 * 2.0 ** -24) + 2.0 ** -20
                got, gl = out[at:at + len(pos), h], lse[at:at + len(pos), h]
                tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.2 * dz[:, None]) * m + 1e-30
                assert (np.abs(got - o) <= tol).all() and (np.abs(gl - l) <= dz + 2.0 ** -22 * np.abs(l)).all(), (layer, s, h)
            at += len(pos)


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
