"""Pins of the page operations' oracle: small written-out cases, and invariants over random sequences of calls."""
import numpy as np

from oracle.pages_oracle import Pool


def test_written_out_case():
    p = Pool(8, 4, 4)
    p.reserve([0, 1], [70, 64])
    assert p.table[0].tolist() == [0, 1, -1, -1] and p.table[1].tolist() == [2, -1, -1, -1]
    p.lens[:2] = 70, 64
    p.fork([0, 0, 1], [2, 3, 2])              # the third names 2 again
    assert p.invalid and p.refs.tolist() == [3, 3, 1, 0, 0, 0, 0, 0]
    p.reserve([2, 0, 3], [1, 1, 1])            # page 1 has three holders, all of which write: the first two get copies
    assert [p.table[s, 1] for s in (2, 0, 3)] == [3, 4, 1] and p.contents[3] == 1 and p.refs[1] == 1
    p.free([0, 1])
    assert p.refs.tolist() == [2, 1, 0, 1, 0, 0, 0, 0]
    assert p.compact() == 3 and p.refs.tolist() == [2, 1, 1, 0, 0, 0, 0, 0] and p.table[2, 1] == 2
    p.check()
    before = p.table.copy()
    p.reserve([2, 3], [64 * 2, 64 * 3])        # the row of 3 is too short: nothing happens for 2 either
    assert p.capacity and np.array_equal(before, p.table)


def test_invariants_under_random_calls():
    rng = np.random.default_rng(0)
    for _ in range(50):
        p = Pool(40, 6, 9)
        for _ in range(60):
            kind = rng.integers(4)
            seqs = rng.permutation(6)[:rng.integers(1, 4)].tolist()
            if kind == 0:
                p.fork(seqs, rng.permutation(6)[:len(seqs)].tolist())
            elif kind == 1:
                n = rng.integers(0, 150, len(seqs)).tolist()
                p.capacity = False
                p.reserve(seqs, n)
                if not p.capacity:
                    for s, k in zip(seqs, n):
                        p.lens[s] += k
                        if k:                  # what is written next is nobody else's
                            assert p.refs[p.table[s, (p.lens[s] - k) // 64]] == 1
            elif kind == 2:
                p.free(seqs[:1])
            else:
                n = p.compact()
                assert (p.refs[:n] > 0).all() and not p.refs[n:].any()
            p.check()


def test_compaction_of_a_wrong_table_moves_nothing():
    for entry in (1, 2, 7, 8):
        p = Pool(8, 3, 4)
        p.reserve([0, 1], [128, 128])
        p.free([0])
        p.table[2, 3] = entry
        before = p.table.copy()
        assert p.compact() == (2 if entry == 2 else 8) and p.invalid == (entry != 2)
        assert np.array_equal(before, p.table) == (entry != 2)


def test_room_in_a_page_that_nobody_holds_is_refused():
    for table, refs, ln, add in (([3, -1], [], 10, 5), ([0, 1], [0], 64, 10), ([0, 1], [0], 20, 100)):
        p = Pool(6, 2, 2)
        p.table[0], p.lens[0] = table, ln
        p.refs[refs] = 1
        p.reserve([0], [add])
        assert p.invalid and p.table[0].tolist() == table and p.refs.sum() == len(refs)
