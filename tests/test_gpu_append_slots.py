"""q4kv_append_slots: the cache holds the bits that q4kv_append makes of the same rows, and nothing else changes."""
import numpy as np
import pytest
import torch

from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV, bits

pytestmark = pytest.mark.gpu


def pools_of(spec, blocks, alias, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    pools = [b.Pool(spec, spec.k_dim, blocks, DEV)] + ([] if alias else [b.Pool(spec, spec.v_dim, blocks, DEV)])
    for p in pools:
        for t in (p.codes, p.scale, p.bias):
            lim = 1 << (31 if t.dtype == torch.int32 else 15)
            t.copy_(torch.randint(-lim, lim, t.shape, generator=g, device=DEV, dtype=t.dtype))
    return pools + ([None] if alias else [])


SHAPES = [(1, 1, 64, 64, False), (2, 8, 128, 128, False), (1, 2, 192, 128, False), (3, 1, 576, 512, True), (2, 3, 64, 320, False), (1, 8, 256, 256, False)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("tokens", [1, 2, 63, 300, 2001])
@pytest.mark.parametrize("kind,fmt,fused", [(torch.float16, b.PARAMS_F16, False), (torch.bfloat16, b.PARAMS_BF16, True), (torch.float16, b.PARAMS_BF16, True),
                                            (torch.bfloat16, b.PARAMS_F16, False)])
def test_same_bits_as_append(shape, tokens, kind, fmt, fused):
    L, H, dk, dv, alias = shape
    if tokens == 2001 and L * H * dk > 600 and fused:
        tokens = 1201
    spec = b.make_spec(L + 1, H, H, dk, dv, alias, param_format=fmt)              # the call's layers begin at 1
    blocks, rng = tokens // 256 + 5, np.random.default_rng(tokens)
    g = torch.Generator(device=DEV).manual_seed(tokens)
    widths = [H * dk] + ([] if alias else [H * dv])
    x = torch.randn((L, tokens, 24 + sum(widths)), generator=g, device=DEV, dtype=kind) * 3
    parts = list(x[..., 24:].split(widths, -1))
    if not fused:
        parts = [p.contiguous() for p in parts]
    rows = [p.unflatten(-1, (H, -1)) for p in parts] + ([None] if alias else [])
    slot = rng.permutation(blocks * 256)[:tokens].astype(np.int32)
    skip = rng.random(tokens) < 0.2
    skip[0] = tokens > 1
    given = slot.copy()
    given[skip] = rng.choice([-1, -256, blocks * 256, 2 ** 31 - 1, -2 ** 31], int(skip.sum()))
    for p in rows:
        if p is not None:                                                       # what has no slot may hold anything
            p[:, torch.from_numpy(skip).to(DEV)] = float("nan")
    kp, vp = pools_of(spec, blocks, alias, 1)
    wk, wv = pools_of(spec, blocks, alias, 1)
    b.q4kv_append_slots(spec, kp, vp, rows[0], rows[1], torch.from_numpy(given).to(DEV), layer_begin=1, layer_end=L + 1)
    # one agent per token: its table names the slot's block, its length the place
    keep = np.flatnonzero(~skip)
    if len(keep):
        at = torch.from_numpy(keep).to(DEV)
        one = [None if p is None else p[:, at].half().contiguous().unsqueeze(2) for p in rows]
        table = torch.from_numpy(slot[keep] // 256).to(DEV).unsqueeze(1).contiguous()
        b.q4kv_append(spec, wk, wv, one[0], one[1], table, torch.from_numpy(slot[keep] % 256).to(DEV), layer_begin=1, layer_end=L + 1)
    torch.cuda.synchronize()
    for p, w in ((kp, wk), (vp, wv)):
        if p is not None:
            for got, want in ((p.codes, w.codes), (p.scale, w.scale), (p.bias, w.bias)):
                assert np.array_equal(bits(got), bits(want))


def test_many_tokens_and_layers():
    """Launches that fill the chip several times over."""
    L, H, dk, tokens = 3, 8, 256, 6000
    spec = b.make_spec(L, H, H, dk)
    g = torch.Generator(device=DEV).manual_seed(0)
    k, v = (torch.randn((L, tokens, H, dk), generator=g, device=DEV, dtype=torch.float16) for _ in range(2))
    kp, vp = pools_of(spec, 24, False, 2)
    wk, wv = pools_of(spec, 24, False, 2)
    slot = torch.arange(tokens, dtype=torch.int32, device=DEV) + 100
    b.q4kv_append_slots(spec, kp, vp, k, v, slot)
    table = torch.arange(24, dtype=torch.int32, device=DEV).unsqueeze(0)
    b.q4kv_append(spec, wk, wv, k.unsqueeze(1), v.unsqueeze(1), table, torch.tensor([100], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for p, w in ((kp, wk), (vp, wv)):
        for got, want in ((p.codes, w.codes), (p.scale, w.scale), (p.bias, w.bias)):
            assert torch.equal(got, want)


def test_no_tokens():
    spec = b.make_spec(1, 1, 1, 64)
    kp, vp = pools_of(spec, 2, False, 3)
    before = kp.codes.clone()
    none = torch.empty((1, 0, 1, 64), dtype=torch.float16, device=DEV)
    b.q4kv_append_slots(spec, kp, vp, none, none, torch.empty(0, dtype=torch.int32, device=DEV))
    b.q4kv_append_slots(spec, kp, vp, none[:0], none[:0], torch.empty(0, dtype=torch.int32, device=DEV), layer_begin=1, layer_end=1)
    torch.cuda.synchronize()
    assert torch.equal(kp.codes, before)


@pytest.mark.parametrize("tokens", [40, 9000])                                    # an octet per group; rounds of 64 groups per wave
def test_one_slot_twice(tokens):
    """Every word in a slot that two tokens have is one of theirs; all other slots hold what they would hold otherwise."""
    spec = b.make_spec(1, 8, 8, 128)
    blocks = tokens // 256 + 2
    g = torch.Generator(device=DEV).manual_seed(tokens)
    k, v = (torch.randn((1, tokens, 8, 128), generator=g, device=DEV, dtype=torch.float16) for _ in range(2))
    first = torch.arange(tokens, dtype=torch.int32, device=DEV)
    both, last = first.clone(), first.clone()
    twice = tokens // 4
    both[-twice:] = first[:twice]                                                 # the last tokens have the first ones' slots
    last[-twice:] = first[:twice]
    last[:twice] = -1
    first[-twice:] = -1
    held = []
    for slot in (both, first, last):
        pools = pools_of(spec, blocks, False, 4)
        b.q4kv_append_slots(spec, *pools, k, v, slot)
        held.append(pools)
    torch.cuda.synchronize()
    for got, one, other in zip(*held):
        for name in ("codes", "scale", "bias"):
            x, y, z = (bits(getattr(p, name)) for p in (got, one, other))
            assert np.all((x == y) | (x == z))
            same = y == z                                                         # slots of one token, and of none
            assert np.array_equal(x[same], y[same]) and not same.all()
