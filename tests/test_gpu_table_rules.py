"""What include/q4kv.h promises of q4kv_resize_tables and q4kv_beam_reorder where blocks, places or rows are missing."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV
from tests.table_rules import PAGE, Rules, families, leave_free, lengths
from tests.test_gpu_block_tables import Both

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("blocks", [1, 4, 1024, 1 << 20])
@pytest.mark.parametrize("places", [0, 3, 5000])
def test_a_table_of_no_rows_needs_no_arrays(blocks, places):
    """Neither table nor lengths nor counts: the map says that there are no tokens, and nobody was refused."""
    refused, begin, slot, agent = ints([77]), ints([77]), torch.full((places + 1,), 77, dtype=torch.int32, device=DEV), ints([77] * (places + 1))
    t = b._CTables(None, None, None, refused.data_ptr(), 0, 7, blocks)
    rc = b.lib().q4kv_resize_tables(C.byref(t), None, places, begin.data_ptr(), slot.data_ptr(), agent.data_ptr(), None, None, None, None, None, 0, b._stream())
    torch.cuda.synchronize()
    assert rc == 0 and refused.item() == 0
    assert begin.item() == (0 if places else 77)
    for x in (slot, agent):
        assert (x[:places] == -1).all() and x[places] == 77


def test_a_reorder_of_no_rows_says_that_nobody_was_refused():
    spec = b.make_spec(1, 1, 1, 64)
    kpool, vpool = b.Pool(spec, 64, 4, DEV), b.Pool(spec, 64, 4, DEV)
    t = b.BlockTables(0, 7, 4, DEV)
    t.refused.fill_(77)
    b.q4kv_beam_reorder(spec, kpool, vpool, t, ints([]))
    torch.cuda.synchronize()
    assert t.refused.item() == 0


class Sides(Both):
    """The same tables and pools on both sides; the model is the header's rule."""

    def __init__(self, table, lens, refs, shape=None, seed=0):
        super().__init__(table, np.array(lens, np.int32), refs, shape, seed)
        self.model = Rules(table, lens, refs, self.model.pools)


PAIR = (2, 1, 64, 128, False)


@pytest.mark.parametrize("shape", [PAIR, None])
def test_a_cut_row_behind_a_refused_one(shape):
    """Blocks are free and places are not: the cut row gets its copy (without pools it has none to get)."""
    table = np.array([[0, -1, -1, -1], [1, 2, -1, -1], [1, 2, -1, -1]], np.int32)
    refs = np.array([1, 2, 2] + [0] * 7, np.int32)
    t = Sides(table, [100, 512, 512], refs, shape)
    t.resize([400, 300, -1], max_tokens=100)
    assert t.model.len == [100, 300 if shape else 256, 512] and t.model.refused == (1 if shape else 2)
    lens = [100, 768, 768]
    table = np.array([[0, -1, -1], [1, 2, 3], [1, 2, 3]], np.int32)
    t = Sides(table, lens, np.array([1, 2, 2, 2] + [0] * 96, np.int32), shape)
    t.resize([110, 700, -1], max_tokens=5)
    assert t.model.len == [100, 700 if shape else 512, 768]


@pytest.mark.parametrize("free", [0, 1])
def test_a_row_left_alone_keeps_its_tokens(free):
    """Somebody else lists the block it ends in, and a row in front of it is refused."""
    table, refs = np.array([[0, -1], [1, 2]], np.int32), np.array([1, 1, 2] + [0] * 5, np.int32)
    refs[3 + free:] = 1
    t = Sides(table, [100, 300], refs, PAIR)
    t.resize([110, -1], max_tokens=5)
    assert t.model.len == [100, 300] and t.model.refused == 1
    t = Sides(table, [100, 300], refs, PAIR)
    t.resize([600, 300], max_tokens=0)
    assert t.model.len == [100, 300] and t.model.refused == 1


def test_a_cut_row_in_front_of_growing_ones_without_blocks():
    """No block for its copy; rows behind it that need none go on."""
    table, refs = np.array([[0, 1], [0, 1], [2, -1], [3, -1]], np.int32), np.array([3, 3, 1, 1, 1], np.int32)
    t = Sides(table, [512, 512, 100, 256], refs, PAIR)
    t.resize([300, -1, 120, 257], max_tokens=100)
    assert t.model.len == [256, 512, 120, 256] and t.model.refused == 2


@pytest.mark.parametrize("rest,places,free,want", [(-1, 100, 0, 120), (-1, 100, 1, 130), (220, 10, 3, 130), (220, 10, 0, 120), (220, 100, 0, 120),
                                                   (220, 100, 1, 130), (220, 100, 3, 130)])
def test_the_row_that_goes_on_overwrites_nobody(rest, places, free, want):
    """Two rows end in one block, the second 80 tokens further on.  Where it stays there, the first goes on in a copy or not at all."""
    table, refs = np.array([[0, -1], [0, -1]], np.int32), np.array([2] + [0] * 3, np.int32)
    refs[1 + free:] = 1
    t = Sides(table, [120, 200], refs, PAIR)
    t.resize([130, rest], max_tokens=places)
    assert t.model.len[0] == want
    if want == 130:
        assert t.model.table[0, 0] != t.model.table[1, 0]


@pytest.mark.parametrize("seed", range(40))
def test_families_of_rows(seed):
    """Rows that list the same blocks and end in them anywhere, few free blocks, few places, rows left alone."""
    rng = np.random.default_rng(seed)
    rows, width = int(rng.choice([3, 9, 40, 600])), int(rng.integers(1, 5))
    table, lens, refs = families(rng, rows, width, members=int(rng.choice([2, 5, 30])))
    if seed % 4:
        leave_free(rng, refs, int(rng.integers(0, 2 + rows // 2)))
    t = Sides(table, lens, refs, PAIR if rows < 100 and seed % 5 else None, seed)
    for _ in range(4):
        t.resize(lengths(rng, t.model.len, width), max_tokens=int(rng.choice([0, 1, 30, 3000, 100000])))


@pytest.mark.parametrize("seed", range(4))
def test_many_families_and_blocks(seed):
    """All rows a table can have, more blocks taken than fit on the chip, and copies among them."""
    rng = np.random.default_rng(seed)
    rows, width = [2048, 1500, 2047, 700][seed], [12, 9, 6, 17][seed]
    table, lens, refs = families(rng, rows, width, members=3)
    if seed == 3:
        leave_free(rng, refs, 4600)
    t = Sides(table, lens, refs, (1, 1, 64, 64, True))
    t.resize([int(n) for n in rng.integers(0, width * PAGE + 1, rows)], max_tokens=0)
    t.resize(lengths(rng, t.model.len, width), max_tokens=2000)
