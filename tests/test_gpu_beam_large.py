"""Beam choices, table calls and ragged appends where offsets pass 2^31, vocabularies have thousands of spans, and two streams are
at it at once."""
import numpy as np
import torch
import pytest

from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV, bits
from tests.test_gpu_beam_select import check, random_rows

pytestmark = pytest.mark.gpu


def test_a_vocabulary_of_millions():
    for kind, num_out in (("f16", 8), ("f32", 64)):
        check(random_rows(1, 2, 3000001, kind), [0.0, -1.0], [0, 2], num_out)


def test_rows_further_apart_than_31_bits():
    """Three rows 1.1 billion elements apart."""
    vocab, stride = 5003, 1100000001
    store = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device=DEV)
    far = store.as_strided((3, vocab), (stride, 1))
    rows = random_rows(2, 3, vocab, "bf16").to(DEV)
    far.copy_(rows)
    score, bounds = torch.tensor([-1.0, -0.5, -0.25], device=DEV), torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    got, want = b.q4kv_beam_select(far, score, bounds, 9), b.q4kv_beam_select(rows, score, bounds, 9)
    torch.cuda.synchronize()
    for x, y in ((got.parent, want.parent), (got.token, want.token), (got.score, want.score)):
        assert torch.equal(x, y)
    assert set(got.parent.view(-1).tolist()) > {2}


def test_blocks_behind_the_second_gigaword_of_a_pool():
    """A latent pool of 9 GB: rows appended into, and a shared last block copied to, its last blocks."""
    blocks, dim = 125003, 576
    spec = b.make_spec(1, 16, 1, dim, 512, True)
    shape = (1, blocks, 1, 256)
    pool = b.Pool.of(torch.empty(shape + (dim // 8,), dtype=torch.int32, device=DEV), torch.empty(shape + (dim // 64,), dtype=torch.int16, device=DEV),
                     torch.empty(shape + (dim // 64,), dtype=torch.int16, device=DEV))
    small = b.Pool(spec, dim, 1, DEV)
    k = torch.randn((1, 256, 1, dim), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=torch.float16)
    last = blocks - 1
    slot = last * 256 + torch.arange(256, dtype=torch.int32, device=DEV)
    for t in (pool.codes, pool.scale, pool.bias):
        t[:, last - 1].fill_(77)
    b.q4kv_append_slots(spec, pool, None, k, None, slot)
    b.q4kv_append_slots(spec, small, None, k, None, slot - last * 256)
    # every block but two is taken; two rows end in the last one, 200 tokens on
    refs = torch.ones(blocks, dtype=torch.int32, device=DEV)
    refs[last], refs[last - 1] = 2, 0
    t = b.BlockTables.of(torch.tensor([[last], [last]], dtype=torch.int32, device=DEV), torch.tensor([200, 200], dtype=torch.int32, device=DEV), refs)
    b.q4kv_beam_reorder(spec, pool, None, t, torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert t.block_table.tolist() == [[last], [last - 1]] and t.refs[-2:].tolist() == [1, 1] and t.refused.item() == 0
    for big, little in ((pool.codes, small.codes), (pool.scale, small.scale), (pool.bias, small.bias)):
        want = bits(little[0, 0])
        assert np.array_equal(bits(big[0, last]), want)
        got = bits(big[0, last - 1])
        assert np.array_equal(got[:, :200], want[:, :200]) and (got[:, 200:] == 77).all()


def test_two_streams_at_once():
    """Calls that share nothing but their inputs, interleaved on two streams."""
    x = [random_rows(s, 24, 40001, "f16").to(DEV) for s in (5, 6)]
    score, bounds = -torch.rand(24, device=DEV), torch.tensor([0, 8, 16, 24], dtype=torch.int32, device=DEV)
    want = [b.q4kv_beam_select(v, score, bounds, 8) for v in x]
    out, work = [b.BeamChoice(3, 8) for _ in x], [b.q4kv_beam_select_workspace(v, 8) for v in x]
    tables = [b.BlockTables(64, 9, 700) for _ in x]
    lens = torch.arange(64, dtype=torch.int32, device=DEV) * 31
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for turn in range(30):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                b.q4kv_beam_select(x[i], score, bounds, 8, out=out[i], workspace=work[i])
                b.q4kv_resize_tables(tables[i], lens if turn % 2 == 0 else lens // 2)
    torch.cuda.synchronize()
    for o, w, t in zip(out, want, tables):
        assert torch.equal(o.parent, w.parent) and torch.equal(o.token, w.token) and torch.equal(o.score, w.score)
        assert t.seq_len.tolist() == (lens // 2).tolist() and int(t.refs.sum()) == sum(-(-n // 256) for n in (lens // 2).tolist())
    assert torch.equal(tables[0].block_table, tables[1].block_table)


def test_a_row_of_one_token_and_groups_of_nothing():
    one = torch.zeros((1, 1), device=DEV)
    got = b.q4kv_beam_select(one, torch.tensor([-2.0], device=DEV), torch.tensor([0, 0, 1, 1], dtype=torch.int32, device=DEV), 3)
    none = b.q4kv_beam_select(one[:0], torch.empty(0, device=DEV), torch.tensor([0, 0, 5], dtype=torch.int32, device=DEV), 2)
    torch.cuda.synchronize()
    assert got.parent.tolist() == [[-1] * 3, [0, -1, -1], [-1] * 3] and got.token.tolist() == [[-1] * 3, [0, -1, -1], [-1] * 3]
    assert got.score[1].tolist() == [-2.0, -float("inf"), -float("inf")]
    assert none.parent.tolist() == [[-1, -1]] * 2 and none.score.tolist() == [[-float("inf")] * 2] * 2
