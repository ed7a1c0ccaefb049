"""q4kv_copy_blocks against indexing on the host, bit for bit, and the flow it serves: agents forked, truncated and
compacted attend as agents that never shared a block."""
import numpy as np
import pytest
import torch

from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV, bits

pytestmark = pytest.mark.gpu


def random_pool(spec, dim, nb, seed):
    p = b.Pool(spec, dim, nb, DEV)
    g = torch.Generator(device=DEV).manual_seed(seed)
    for t in (p.codes, p.scale, p.bias):
        lim = 1 << (31 if t.dtype == torch.int32 else 15)
        t.copy_(torch.randint(-lim, lim, t.shape, generator=g, device=DEV, dtype=t.dtype))
    return p


@pytest.mark.parametrize("shape", [(1, 1, 64, 64, False, 3, 1), (3, 2, 192, 128, False, 9, 4), (2, 1, 576, 512, True, 20, 7), (5, 8, 256, 256, False, 8, 3),
                                   (2, 3, 64, 320, False, 40, 19)])
def test_pairs_are_copied_and_nothing_else_changes(shape):
    L, H, dk, dv, alias, nb, n = shape
    spec = b.make_spec(L, H, H, dk, dv, alias)
    pools = [random_pool(spec, dk, nb, 1)] + ([] if alias else [random_pool(spec, dv, nb, 2)])
    ids = np.random.default_rng(n).permutation(nb).astype(np.int32)
    src, dst = ids[:n].copy(), ids[n:2 * n].copy()
    if n > 3:
        src[2] = src[0]                                                  # one source of two copies
        src[3], dst[1] = nb, -1                                          # ids outside the pool: skipped
    src, dst = np.append(src, ids[-1]), np.append(dst, ids[-1])          # a block onto itself: skipped
    want = [[bits(t).copy() for t in (p.codes, p.scale, p.bias)] for p in pools]
    for s, d in zip(src, dst):
        if 0 <= s < nb and 0 <= d < nb:
            for w in want:
                for t in w:
                    t[:, d] = t[:, s]
    b.q4kv_copy_blocks(spec, pools[0], None if alias else pools[1], torch.from_numpy(src).to(DEV), torch.from_numpy(dst).to(DEV))
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        for t, x in zip((p.codes, p.scale, p.bias), w):
            assert np.array_equal(bits(t), x)


def test_more_pairs_than_a_launch_has_rows():
    spec = b.make_spec(1, 1, 1, 64)
    pools = [random_pool(spec, 64, 4, i) for i in (1, 2)]
    n = 70001
    src, dst = np.full(n, -1, np.int32), np.zeros(n, np.int32)
    src[0], dst[0], src[-1], dst[-1] = 2, 0, 3, 1
    want = [t.codes.clone() for t in pools]
    for w in want:
        w[:, 0], w[:, 1] = w[:, 2], w[:, 3]
    b.q4kv_copy_blocks(spec, *pools, torch.from_numpy(src).to(DEV), torch.from_numpy(dst).to(DEV))
    torch.cuda.synchronize()
    assert all(torch.equal(p.codes, w) for p, w in zip(pools, want))


def test_no_pairs_and_pairs_that_do_not_match():
    spec = b.make_spec(1, 1, 1, 64)
    pools = [random_pool(spec, 64, 2, i) for i in (1, 2)]
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    b.q4kv_copy_blocks(spec, *pools, none, none)
    with pytest.raises(ValueError):
        b.q4kv_copy_blocks(spec, *pools, none, torch.zeros(1, dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        b.q4kv_copy_blocks(spec, *pools, none.long(), none.long())


def test_on_a_side_stream_and_captured():
    spec = b.make_spec(2, 2, 2, 128)
    pools = [random_pool(spec, 128, 6, i) for i in (1, 2)]
    src, dst = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, 1], [4, 3]))
    want = [(p.codes[:, [0, 1]].clone(), p.bias[:, [0, 1]].clone()) for p in pools]

    def check():
        torch.cuda.synchronize()
        for p, (c, x) in zip(pools, want):
            assert torch.equal(p.codes[:, [4, 3]], c) and torch.equal(p.bias[:, [4, 3]], x)
            p.codes[:, 3:5] = 0
            p.bias[:, 3:5] = 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.q4kv_copy_blocks(spec, *pools, src, dst)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.q4kv_copy_blocks(spec, *pools, src, dst)
    for _ in range(3):
        graph.replay()
        check()


def test_forked_and_compacted_agents_attend_as_if_they_never_shared():
    """A parent's cache, two children at different points, each then writes tokens of its own; one is cut back; the pool is
    compacted.  Every agent's attention equals that of an agent whose whole cache was appended into blocks of its own."""
    L, Hq, Hkv, D = 2, 8, 2, 128
    spec = b.make_spec(L, Hq, Hkv, D)
    rng = np.random.default_rng(8)
    rows = lambda n: [torch.from_numpy(rng.standard_normal((L, 1, n, Hkv, D)).astype(np.float16)).to(DEV) for _ in range(2)]  # noqa: E731
    book, NB = b.BlockPool(24), 24
    pools = [b.Pool(spec, D, NB, DEV, True) for _ in range(2)]
    history = {}                                                         # agent -> list of (K rows, V rows)

    def length(a):
        return sum(k.shape[2] for k, _ in history[a])

    def table(a):
        return torch.tensor([book.table_row(a, 8, 0)], dtype=torch.int32, device=DEV)

    def write(a, n):
        k, v = rows(n)
        before = torch.tensor([length(a)], dtype=torch.int32, device=DEV)
        book.reserve(a, length(a) + n)
        b.q4kv_append(spec, *pools, k, v, table(a), before)
        history[a].append((k, v))

    def copy(pairs):
        if pairs:
            b.q4kv_copy_blocks(spec, *pools, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in zip(*pairs)))

    def cut(a, n):
        k, v = (torch.cat([r[i] for r in history[a]], 2)[:, :, :n].contiguous() for i in (0, 1))
        return [(k, v)]
    history[0] = []
    write(0, 700)
    for child, n in ((1, 700), (2, 512), (3, 100)):
        copy(book.fork(0, child, n))
        history[child] = cut(0, n)
        write(child, 90 + child)
    write(0, 33)
    copy(book.truncate(1, 300))
    history[1] = cut(1, 300)
    write(1, 5)
    book.release(0)
    copy(book.compact())
    write(2, 300)
    q = torch.from_numpy(rng.standard_normal((L, 1, 1, Hq, D)).astype(np.float16)).to(DEV)
    for a in (1, 2, 3):
        n = length(a)
        (k, v), = cut(a, n)
        alone = [b.Pool(spec, D, 8, DEV, True) for _ in range(2)]
        own = torch.arange(8, dtype=torch.int32, device=DEV)[None].contiguous()
        b.q4kv_append(spec, *alone, k, v, own, torch.zeros(1, dtype=torch.int32, device=DEV))
        sl = torch.tensor([n], dtype=torch.int32, device=DEV)
        got = b.q4kv_batched_attention(spec, *pools, q, table(a), sl, n, 0.09)
        want = b.q4kv_batched_attention(spec, *alone, q, own, sl, n, 0.09)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.isfinite(want).all()
