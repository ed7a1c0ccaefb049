"""q4kv_resize_tables and q4kv_beam_reorder against a row-by-row model, all integers equal: tables, lengths, counts, slot maps,
and every byte of the pools."""
import numpy as np
import pytest
import torch

from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV, bits
from tests.table_model import PAGE, Tables, blocks_of

pytestmark = pytest.mark.gpu


def state(rng, lens, max_blocks, num_blocks, share=1, outside=0):
    """Rows of these lengths with shuffled blocks; families of `share` rows list the whole blocks of their shortest row together;
    `outside` blocks belong to somebody else."""
    ids = list(rng.permutation(num_blocks))
    table, refs = np.full((len(lens), max_blocks), -1, np.int32), np.zeros(num_blocks, np.int32)
    for f in range(0, len(lens), share):
        common = [ids.pop() for _ in range(min(lens[f:f + share]) // PAGE)] if share > 1 else []
        for r in range(f, min(f + share, len(lens))):
            mine = common + [ids.pop() for _ in range(blocks_of(lens[r]) - len(common))]
            table[r, :len(mine)] = mine
            refs[mine] += 1
    for _ in range(min(outside, len(ids))):
        refs[ids.pop()] = 1
    return table, np.array(lens, np.int32), refs


class Both:
    """The same tables and pools on both sides."""

    def __init__(self, table, lens, refs, shape=None, seed=0):
        self.spec, self.pools, host = None, (None, None), None
        if shape is not None:
            L, H, dk, dv, alias = shape
            self.spec = b.make_spec(L, H, H, dk, dv, alias)
            g = torch.Generator(device=DEV).manual_seed(seed)
            pools = [b.Pool(self.spec, d, len(refs), DEV) for d in ([dk] if alias else [dk, dv])]
            for p in pools:
                for t in (p.codes, p.scale, p.bias):
                    lim = 1 << (31 if t.dtype == torch.int32 else 15)
                    t.copy_(torch.randint(-lim, lim, t.shape, generator=g, device=DEV, dtype=t.dtype))
            self.arrays = [t for p in pools for t in (p.codes, p.scale, p.bias)]
            host = [bits(t).copy() for t in self.arrays]
            self.pools = (pools[0], None if alias else pools[1])
        self.model = Tables(table, lens, refs, host)
        self.t = b.BlockTables.of(*(torch.from_numpy(x.copy()).to(DEV) for x in (table, lens, refs)))

    def args(self):
        return dict(spec=self.spec, kpool=self.pools[0], vpool=self.pools[1])

    def check(self):
        torch.cuda.synchronize()
        assert self.t.seq_len.tolist() == self.model.len
        for r, n in enumerate(self.model.len):
            assert self.t.block_table[r, :blocks_of(n)].tolist() == self.model.table[r, :blocks_of(n)].tolist(), r
        assert np.array_equal(self.t.block_table.cpu().numpy(), self.model.table)
        assert np.array_equal(self.t.refs.cpu().numpy(), self.model.refs)
        assert self.t.refused.item() == self.model.refused
        if self.spec is not None:
            for got, want in zip(self.arrays, self.model.pools):
                assert np.array_equal(bits(got), want)

    def resize(self, new_len, max_tokens=0, slack=3):
        out = None
        if max_tokens:
            out = b.TokenMap(self.t, max_tokens + slack)
            for x in (out.begin, out.slot, out.agent, out.position):
                x.fill_(-77)
            whole = out.slot, out.agent, out.position
            out.slot, out.agent, out.position = (x[:max_tokens] for x in whole)
        want = self.model.resize(new_len, max_tokens)
        b.q4kv_resize_tables(self.t, torch.tensor(new_len, dtype=torch.int32, device=DEV), out=out, **self.args())
        self.check()
        if max_tokens:
            for got, w in zip((out.begin, out.slot, out.agent, out.position), want):
                assert got.tolist() == list(w)
            assert all((x[max_tokens:] == -77).all() for x in whole)

    def reorder(self, parent):
        self.model.reorder(parent)
        b.q4kv_beam_reorder(self.spec, *self.pools, self.t, torch.tensor(parent, dtype=torch.int32, device=DEV))
        self.check()


@pytest.mark.parametrize("rows,blocks,hi,seed", [(1, 5, 300, 0), (3, 40, 1000, 1), (40, 900, 6000, 2), (257, 3000, 2500, 3), (1025, 5001, 900, 4),
                                                 (2048, 16383, 1500, 5), (64, 17000, 60000, 6)])
def test_lengths_grow_and_shrink(rows, blocks, hi, seed):
    rng = np.random.default_rng(seed)
    width = blocks_of(hi) + 1
    lens = [int(n) for n in rng.integers(0, hi, rows)]
    used = sum(map(blocks_of, lens))
    t = Both(*state(rng, lens, width, max(blocks, used + 1), outside=rows // 3))
    for step in range(3):
        new = [int(n) for n in rng.integers(0, hi, rows)]
        for r in range(rows):                   # some rows stay, some are left alone, some want more than their table lists
            new[r] = [new[r], t.model.len[r], -5, width * PAGE + 1][int(rng.choice(4, p=[0.7, 0.1, 0.1, 0.1]))]
        t.resize(new, max_tokens=int(rng.integers(1, 1 + max(1, rows * hi // 4))) if step != 1 else 0)
    t.resize([0] * rows)
    assert (t.t.block_table == -1).all()


def test_one_token_at_a_time_over_the_ends_of_blocks():
    rng = np.random.default_rng(0)
    t = Both(*state(rng, [0, 1, 255, 256, 257, 510, 511, 512], 5, 31))
    for _ in range(4):
        t.resize([n + 1 for n in t.model.len], max_tokens=8)
    for _ in range(6):
        t.resize([max(0, n - 1) for n in t.model.len], max_tokens=8)


@pytest.mark.parametrize("free,places", [(0, 100), (1, 100), (2, 100), (3, 100), (4, 100), (50, 1), (50, 9), (50, 10), (50, 11), (50, 300), (50, 100000)])
def test_rows_behind_the_first_that_cannot_be_served(free, places):
    """Blocks or places run out in the middle: what is in front is served, what is behind is not, rows that shrink are."""
    rng = np.random.default_rng(free + places)
    lens = [250, 300, 256, 900, 10, 0, 512]
    table, l, refs = state(rng, lens, 9, 200)
    unused = np.flatnonzero(refs == 0)
    refs[unused[free:]] = 1
    t = Both(table, l, refs)
    t.resize([259, 301, 600, 900, 4, 700, 530], max_tokens=places)


def test_more_blocks_than_fit_on_chip_are_taken():
    rng = np.random.default_rng(8)
    table, lens, refs = state(rng, [100, 0, 0, 300], 9000, 20011, outside=3001)
    t = Both(table, lens, refs)
    t.resize([4500 * PAGE + 3, 7, 5000 * PAGE, 300], max_tokens=0)
    t.resize([0, 4000 * PAGE, 0, 2 ** 31 - 1], max_tokens=4000 * PAGE)


SHAPES = [(1, 1, 64, 64, False), (3, 2, 192, 128, False), (2, 1, 576, 512, True), (2, 3, 64, 320, False), (1, 8, 256, 256, False)]


@pytest.mark.parametrize("shape", SHAPES)
def test_beams_take_their_parents_rows(shape):
    rng = np.random.default_rng(shape[2])
    beams = 5
    lens = [n for n in (700, 513, 512, 40, 255) for _ in range(beams)]
    t = Both(*state(rng, lens, 4, 85, share=beams), shape=shape)
    for step in range(4):
        parent = [f + int(rng.integers(0, beams)) for f in range(0, len(lens), beams) for _ in range(beams)]
        t.reorder(parent)
        t.resize([n + int(rng.integers(0, 2)) * (step % 2) + 3 * (step // 2) for n in t.model.len], max_tokens=100)


@pytest.mark.parametrize("parent", [[0, 0, 0, 0], [3, 2, 1, 0], [1, 1, 3, 3], [-1, 0, 99, 2], [2, 2, 2, -7], [1, 2, 3, 0], [0, 1, 2, 3], [4, 4, 4, 4]])
@pytest.mark.parametrize("lens", [[0, 0, 0, 0], [1, 300, 256, 511], [800, 800, 800, 800], [257, 0, 40, 1000]])
def test_any_parents(parent, lens):
    rng = np.random.default_rng(1)
    t = Both(*state(rng, lens, 5, 40, share=2), shape=(2, 1, 64, 64, False))
    t.reorder(parent)
    t.reorder(parent)


@pytest.mark.parametrize("rows,width,seed", [(8, 1500, 0), (300, 40, 1), (2048, 9, 2), (2047, 17, 3), (1, 3, 4), (33, 1025, 5)])
def test_tables_of_many_rows_and_columns(rows, width, seed):
    """More entries than one workgroup holds; also rows in one family with a wide shared prefix."""
    rng = np.random.default_rng(seed)
    lens = [int(n) for n in rng.integers(0, width * PAGE, rows)]
    lens[0] = width * PAGE
    share = 1 if seed % 2 else 4
    t = Both(*state(rng, lens, width, sum(map(blocks_of, lens)) + rows // 2 + 1, share=share), shape=(1, 1, 64, 64, True))
    t.reorder([int(p) for p in rng.integers(-1, rows + 1, rows)])
    t.reorder([int(p) for p in np.sort(rng.integers(0, rows, rows))])


@pytest.mark.parametrize("free", [0, 1, 2, 5])
def test_no_block_left_for_a_copy(free):
    rng = np.random.default_rng(free)
    table, lens, refs = state(rng, [300, 300, 300, 300], 3, 40, share=4)
    refs[np.flatnonzero(refs == 0)[free:]] = 1
    t = Both(table, lens, refs, shape=(1, 2, 64, 64, False))
    t.reorder([2, 2, 2, 2])                     # three blocks come free, three are needed
    t.reorder([1, 1, 0, -1])


def test_cut_inside_a_shared_block():
    """With pools the first tokens are copied; rows that all end in a block leave it to the lowest; without pools the row goes
    back to the full blocks."""
    rng = np.random.default_rng(5)
    for shape in ((2, 1, 128, 64, False), None):
        t = Both(*state(rng, [1030, 1100, 1200, 1024, 900, 900], 6, 60, share=3), shape=shape)
        t.resize([700, 1100, 1200, 1024, 300, -1], max_tokens=5)
        t.resize([700, 600, 600, 1030, 300, 299], max_tokens=50)
        t.resize([1, 1, 1, 0, 2, 2], max_tokens=50)


def test_a_row_goes_on_in_a_block_that_others_list():
    """Rows made alike by hand (copied entries, counted twice): the growing rows get copies first."""
    rng = np.random.default_rng(6)
    table, lens, refs = state(rng, [600, 0, 0, 300], 5, 30)
    table[1], table[2] = table[0], table[0]
    lens[1] = lens[2] = 600
    refs[table[0, :3]] += 2
    t = Both(table, lens, refs, shape=(1, 2, 64, 128, False))
    t.resize([601, 601, -1, 301], max_tokens=9)


def test_counts_and_entries_that_are_no_blocks():
    """Entries outside the pool are carried along and counted nowhere; lengths outside the table are read as its ends."""
    rng = np.random.default_rng(7)
    table, lens, refs = state(rng, [700, 300, 40], 4, 20)
    table[0, 1], table[1, 1] = 20, -3
    t = Both(table, lens, refs, shape=(1, 1, 64, 64, True))
    t.reorder([1, 0, 0])
    t.resize([10, 710, 0], max_tokens=900)
    t.t.seq_len.copy_(torch.tensor([-9, 10 ** 9, 3]))
    t.model.len = [0, 4 * PAGE, 3]
    t.model.table[0], t.model.table[1] = t.t.block_table[0].tolist(), t.t.block_table[1].tolist()
    t.resize([0, 700, 3], max_tokens=7)


def test_nothing_to_do():
    t = Both(*state(np.random.default_rng(0), [], 3, 9))
    out = b.TokenMap(t.t, 4)
    out.slot.fill_(5)
    b.q4kv_resize_tables(t.t, torch.zeros(0, dtype=torch.int32, device=DEV), out=out)
    torch.cuda.synchronize()
    assert out.begin.tolist() == [0] and out.slot.tolist() == [-1] * 4
