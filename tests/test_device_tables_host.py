"""Refusals of q4kv_append_slots, q4kv_resize_tables, q4kv_beam_reorder and q4kv_beam_select: found on the host, before any launch."""
import ctypes as C
import re

import pytest
import torch

from paper_2603_04428_amd import binding as b


def err():
    return b.lib().q4kv_last_error().decode()


def pool(blocks=4):
    return b._CPool(0x1000, 0x2000, 0x3000, blocks)


SPEC = b.make_spec(2, 4, 2, 128)
LATENT = b.make_spec(2, 16, 1, 576, 512, True)


def slots(spec=SPEC, k=None, v=False, **kw):
    a = dict(k_new=0x4000, v_new=0x5000, fmt=0, ks=256, vs=256, slot=0x6000, n=5, lb=0, le=2)
    a.update(kw)
    k, v = k or pool(), pool() if v is False else v
    return b.lib().q4kv_append_slots(C.byref(spec), C.byref(k), None if v is None else C.byref(v), a["k_new"], a["v_new"], a["fmt"], a["ks"],
                                     a["vs"], a["slot"], a["n"], a["lb"], a["le"], None)


@pytest.mark.parametrize("code,text,kw", [
    (-1, "V pool", dict(v=None)), (-1, "num_blocks", dict(v=pool(5))), (-1, "in_format", dict(fmt=2)), (-1, "layer range", dict(le=3)),
    (-1, "layer range", dict(lb=2, le=1)), (-1, "negative", dict(n=-1)), (-3, "pieces", dict(n=(1 << 20) + 1)),
    (-3, "31 bits", dict(k=pool(1 << 23), v=pool(1 << 23))), (-1, "NULL", dict(k_new=None)), (-1, "NULL", dict(v_new=None)),
    (-1, "NULL", dict(slot=None)), (-1, "aligned", dict(k_new=0x4008)), (-1, "aligned", dict(v_new=0x5002)), (-2, "strides", dict(ks=248)),
    (-2, "strides", dict(vs=260)), (-2, "strides", dict(ks=-256)), (-1, "NULL when", dict(spec=LATENT, v=None, ks=576)),
    (-1, "NULL when", dict(spec=LATENT, v_new=None, ks=576)), (-3, "2\\^31", dict(spec=b.make_spec(1, 128, 128, 1024), n=1 << 20, ks=1 << 17, vs=1 << 17, le=1))])
def test_append_slots_refusals(code, text, kw):
    assert slots(**kw) == code
    assert re.search(text, err())


def test_append_slots_with_nothing_to_do():
    assert slots(n=0, k_new=None, v_new=None, slot=None) == 0
    assert slots(lb=1, le=1, k_new=None) == 0


def tables(**kw):
    a = dict(block_table=0x4000, seq_len=0x5000, refs=0x6000, refused=None, num_agents=3, max_blocks=7, num_blocks=4)
    a.update(kw)
    return b._CTables(**a)


def resize(t=None, spec=None, k=None, v=None, **kw):
    a = dict(new=0x7000, n=10, begin=0x8000, slot=0x9000, agent=None, position=None, ws=0xA000, bytes=1 << 20)
    a.update(kw)
    t = t or tables()
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return b.lib().q4kv_resize_tables(ref(t), a["new"], a["n"], a["begin"], a["slot"], a["agent"], a["position"], ref(spec), ref(k), ref(v), a["ws"],
                                      a["bytes"], None)


def reorder(t=None, spec=SPEC, k=None, v=None, parent=0x7000, ws=0xA000, n=1 << 20):
    t, k, v = t or tables(), k or pool(), v or pool()
    return b.lib().q4kv_beam_reorder(C.byref(spec), C.byref(k), C.byref(v), C.byref(t), parent, ws, n, None)


BAD_TABLES = [(-1, "negative", dict(num_agents=-1)), (-1, "negative", dict(max_blocks=0)), (-1, "negative", dict(num_blocks=0)),
              (-3, "2049 rows", dict(num_agents=2049)), (-3, "31 bits", dict(num_blocks=1 << 23)), (-3, "2\\^31 tokens", dict(max_blocks=(1 << 23) + 1)),
              (-1, "NULL", dict(block_table=None)), (-1, "NULL", dict(seq_len=None)), (-1, "NULL", dict(refs=None)), (-1, "aligned", dict(refs=0x6004))]


@pytest.mark.parametrize("code,text,kw", BAD_TABLES)
def test_tables_refusals(code, text, kw):
    for call in (resize, reorder):
        assert call(t=tables(**kw)) == code
        assert re.search(text, err())


@pytest.mark.parametrize("code,text,kw", [
    (-1, "negative", dict(n=-1)), (-1, "NULL", dict(new=None)), (-1, "map", dict(slot=None)), (-1, "map", dict(begin=None)),
    (-1, "without a spec", dict(k=pool())), (-1, "K pool", dict(spec=SPEC)), (-1, "V pool", dict(spec=SPEC, k=pool())),
    (-1, "tables of 4 blocks, pools of 5", dict(spec=SPEC, k=pool(5), v=pool(5))), (-4, "workspace", dict(spec=SPEC, k=pool(), v=pool(), ws=None)),
    (-4, "workspace", dict(spec=SPEC, k=pool(), v=pool(), bytes=100)), (-1, "aligned", dict(spec=SPEC, k=pool(), v=pool(), ws=0xA008)),
    (-1, "NULL when", dict(spec=LATENT, k=pool(), v=pool()))])
def test_resize_refusals(code, text, kw):
    assert resize(**kw) == code and text in err()


def test_reorder_refusals():
    assert reorder(parent=None) == -1 and "NULL" in err()
    assert reorder(ws=None) == -4
    assert reorder(n=b.lib().q4kv_tables_workspace_bytes(3) - 1) == -4
    assert reorder(k=pool(9), v=pool(9)) == -1 and "pools of 9" in err()
    assert reorder(t=tables(num_agents=0, block_table=None, seq_len=None, refs=None), parent=None) == 0
    assert b.lib().q4kv_tables_workspace_bytes(-1) == 0 and b.lib().q4kv_tables_workspace_bytes(2049) == 0
    assert b.lib().q4kv_tables_workspace_bytes(2048) > b.lib().q4kv_tables_workspace_bytes(1) > 0


def select(**kw):
    a = dict(logits=0x4000, fmt=0, stride=1000, vocab=1000, rows=4, score=0x5000, end=None, bounds=0x6000, groups=2, out=2, parent=0x7000,
             token=0x8000, total=0x9000, ws=0xA000, bytes=1 << 30)
    a.update(kw)
    return b.lib().q4kv_beam_select(*a.values(), None)


@pytest.mark.parametrize("code,text,kw", [
    (-1, "logits_format", dict(fmt=3)), (-1, "logits_format", dict(fmt=-1)), (-1, "negative", dict(vocab=0)), (-1, "negative", dict(rows=-1)),
    (-1, "negative", dict(groups=-1)), (-3, "groups", dict(groups=1 << 22)), (-3, "fewer groups", dict(rows=1 << 23, vocab=1 << 18, stride=1 << 18)), (-3, "vocabulary", dict(vocab=(1 << 30) + 1, stride=1 << 40)), (-3, "num_out", dict(out=0)), (-3, "num_out", dict(out=65)),
    (-3, "fewer groups", dict(rows=2 ** 31 - 1, vocab=1 << 20, stride=1 << 20)), (-2, "apart", dict(stride=999)), (-1, "NULL", dict(logits=None)),
    (-1, "NULL", dict(score=None)), (-1, "NULL", dict(bounds=None)), (-1, "NULL", dict(parent=None)), (-1, "NULL", dict(token=None)),
    (-1, "NULL", dict(total=None)), (-1, "element", dict(logits=0x4001)), (-1, "element", dict(logits=0x4002, fmt=2)), (-4, "workspace", dict(ws=None)),
    (-4, "workspace", dict(bytes=64)), (-1, "aligned", dict(ws=0xA008))])
def test_select_refusals(code, text, kw):
    assert select(**kw) == code and text in err()


def test_select_sizes():
    assert select(groups=0, bounds=None, parent=None, token=None, total=None) == 0
    need = b.lib().q4kv_beam_select_workspace_bytes
    assert need(0, 1000, 4, 2) >= 4 * 24
    assert need(3, 1000, 4, 2) == 0 and need(0, 0, 4, 2) == 0 and need(0, 1000, -1, 2) == 0 and need(0, 1000, 4, 65) == 0
    assert need(2, 1000, 0, 2) >= 16


def test_binding_refuses_what_the_library_cannot_see():
    cpu = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        b.q4kv_beam_select(cpu, torch.zeros(4), torch.zeros(2, dtype=torch.int32), 1)
    t = b.BlockTables(3, 4, 5, device="cpu")
    with pytest.raises(TypeError):
        b.q4kv_resize_tables(t, torch.zeros(3, dtype=torch.int32))
    t.seq_len = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        t.c()
    spec = b.make_spec(1, 1, 1, 64)
    with pytest.raises(TypeError):
        b.q4kv_append_slots(spec, None, None, torch.zeros(1, 3, 64, dtype=torch.float16), None, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        b.q4kv_append_slots(spec, None, None, torch.zeros(1, 3, 1, 64, dtype=torch.float16), None, torch.zeros(3, dtype=torch.int32))
