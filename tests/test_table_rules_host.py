"""The model of q4kv_resize_tables in tests/table_rules.py keeps what include/q4kv.h promises, whatever rows share."""
import numpy as np
import pytest

from tests.table_model import PAGE, blocks_of
from tests.table_rules import Rules, families, leave_free, lengths


def texts(t):
    """What every row reads: one number per token."""
    pool = t.pools[0][0, :, 0, :, 0]
    return [np.concatenate([pool[t.table[r, j]] for j in range(blocks_of(n))] or [np.zeros(0, int)])[:n].tolist() for r, n in enumerate(t.len)]


def listings(t):
    n = np.zeros_like(t.refs)
    for r, length in enumerate(t.len):
        n[t.table[r, :blocks_of(length)]] += 1
    return n


@pytest.mark.parametrize("seed", range(60))
def test_no_row_loses_or_overwrites_anything_it_need_not(seed):
    rng = np.random.default_rng(seed)
    rows, width = int(rng.integers(1, 14)), int(rng.integers(1, 5))
    table, lens, refs = families(rng, rows, width)
    if seed % 3:
        leave_free(rng, refs, int(rng.integers(0, 7)))
    pool = rng.integers(0, 1 << 40, (1, len(refs), 1, PAGE, 1))
    t = Rules(table, lens, refs, [pool])
    for step in range(4):
        before, old, outside, unused = texts(t), list(t.len), t.refs - listings(t), t.refs == 0
        new = lengths(rng, t.len, width)
        places = int(rng.choice([0, 1, 5, 100, 100000]))
        begin, slot, agent, position = t.resize(new, places)
        assert np.array_equal(t.refs - listings(t), outside) and (t.refs >= 0).all()
        refused, stopped = 0, False
        for r in range(rows):
            want = old[r] if new[r] < 0 or new[r] > width * PAGE else new[r]
            refused += new[r] > width * PAGE
            if want > old[r]:
                assert t.len[r] in (old[r], want) and not (stopped and t.len[r] == want)
                stopped |= t.len[r] == old[r]
                refused += t.len[r] == old[r]
            elif t.len[r] != want:
                assert want < old[r] and want % PAGE and t.len[r] == want // PAGE * PAGE
                assert not (unused & (t.refs == 0)).any(), "a block is left"
                refused += 1
        assert t.refused == refused
        # new tokens go where nobody else has any, and every row still reads its own
        mine = {}
        for r, n in enumerate(t.len):
            for p in range(min(n, old[r])):
                mine.setdefault((int(t.table[r, p // PAGE]), p % PAGE), []).append(r)
        new_tokens = [(r, p) for r, n in enumerate(t.len) for p in range(old[r], n)]
        written = [(int(t.table[r, p // PAGE]), p % PAGE) for r, p in new_tokens]
        assert len(set(written)) == len(written)
        assert not any(set(mine.get(w, [])) for w in written)
        for k, (block, place) in enumerate(written):
            t.pools[0][0, block, 0, place, 0] = seed * 10000 + step * 1000 + k
        after = texts(t)
        for r in range(rows):
            n = min(len(before[r]), len(after[r]))
            assert after[r][:n] == before[r][:n]
        if places:
            assert [s for s in slot if s >= 0] == [b * PAGE + i for b, i in written] and begin[-1] == len(written)


def test_a_cut_row_gets_its_copy_behind_a_refused_one():
    """Blocks are free; the row in front wants more places than the map has."""
    table = np.array([[0, -1, -1, -1], [1, 2, -1, -1], [1, 2, -1, -1]], np.int32)
    refs = np.array([1, 2, 2] + [0] * 7, np.int32)
    t = Rules(table, [100, 512, 512], refs, [np.zeros((1, 10, 1, PAGE, 1), int)])
    t.resize([400, 300, -1], 100)
    assert t.len == [100, 300, 512] and t.refused == 1


def test_a_row_left_alone_behind_a_refused_one_keeps_its_tokens():
    """Somebody else lists its last block."""
    t = Rules(np.array([[0, -1], [1, 2]], np.int32), [100, 300], np.array([1, 1, 2] + [0] * 5, np.int32), [np.zeros((1, 8, 1, PAGE, 1), int)])
    t.resize([110, -1], 5)
    assert t.len == [100, 300] and t.refused == 1
