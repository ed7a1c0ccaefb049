"""The step between two decode calls, measured: what batches of requests and beams need so that their bookkeeping stays on the GPU.

Four kinds of case:
  select   a beam step's choice: log-softmax of every row of logits, plus the row's score; of all continuations of a group's rows
           the best num_out, ties to the lowest row, then token (q4kv_beam_select)
  reorder  rows of the block table become copies of their parents' rows: blocks are counted, and the last, partly filled block of a
           parent with several children is copied for all of them but the first (q4kv_beam_reorder)
  tables   requests grow to new lengths: free blocks are taken, lowest id first, and every new token gets its slot, agent and
           position; then they are cut back to the old lengths, and the blocks are free again (q4kv_resize_tables, twice)
  append   ragged new tokens of all requests quantized into the slots of such a map (q4kv_append_slots); the pages are then read
           back (q4kv_dequantize), which is part of the pass

A cache row is cut into groups of 64 values; a group stores bias = min, scale = (max - min) / 15 and eight 4-bit codes a word.
A slot is block * 256 + place in the block.
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 64
PAGE = 256

# head shapes: query heads, KV heads, key width, value width, V is a prefix of K
SHAPES = {
    "llama": (32, 8, 128, 128, False),      # Llama-3.1-8B-shaped: four query heads per KV head
    "gemma": (16, 8, 256, 256, False),      # Gemma-3-12B-shaped: two
    "latent": (16, 1, 576, 512, True),      # DeepSeek-V2-Lite-shaped shared latent: sixteen on one row
    "per_head": (16, 16, 192, 128, False),  # the same model's decompressed per-head cache
    "narrow": (8, 1, 64, 64, False),        # 64-wide heads, eight query heads on one KV head
}
KINDS = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one request of four beams, a small vocabulary: latency
        dict(name="select_1x4_32k", kind="select", groups=1, beams=4, ragged=False, vocab=32000, pad=0, out=4, type="f16", banned=0.0, finished=0.0),
        # the first step: all beams start from one row, the others are dead; eight are wanted of a large vocabulary
        dict(name="select_first_10x8_128k", kind="select", groups=10, beams=8, ragged=False, vocab=128000, pad=0, out=8, type="bf16", banned=0.0, finished=-1.0),
        # twice as many candidates as beams, an odd vocabulary whose rows lie an odd stride apart, a grammar that bans most tokens
        dict(name="select_16x8_odd", kind="select", groups=16, beams=8, ragged=True, vocab=50001, pad=2, out=16, type="f32", banned=0.7, finished=0.2),
        # a full batch over the largest vocabulary
        dict(name="select_64x4_262k", kind="select", groups=64, beams=4, ragged=False, vocab=262144, pad=0, out=4, type="bf16", banned=0.0, finished=0.05),
        # one request's four beams, two of them gone
        dict(name="reorder_llama_1x4", kind="reorder", shape="llama", layers=32, groups=1, beams=4, prompt=1500, made=37, bf16=False),
        # ten requests' beams
        dict(name="reorder_gemma_10x4", kind="reorder", shape="gemma", layers=48, groups=10, beams=4, prompt=700, made=150, bf16=False),
        # wide beams of four requests on latent rows, far into the text
        dict(name="reorder_latent_4x16", kind="reorder", shape="latent", layers=27, groups=4, beams=16, prompt=3000, made=901, bf16=True),
        # a decode step: every request gets its next token, one in 256 a new block; latency
        dict(name="tables_step_40", kind="tables", agents=40, share=4, lo=300, hi=8000, grow_lo=1, grow_hi=1, slack=600, pad=0),
        # drafts of one to nine tokens are given places and taken back
        dict(name="tables_drafts_500", kind="tables", agents=500, share=1, lo=1, hi=6000, grow_lo=1, grow_hi=9, slack=9000, pad=300),
        # a full batch of prompts is admitted, and released
        dict(name="tables_admit_400", kind="tables", agents=400, share=1, lo=0, hi=0, grow_lo=3, grow_hi=1400, slack=20000, pad=0),
        # one decode token of each request and two short prompts, one layer's call
        dict(name="append_gemma_step", kind="append", shape="gemma", layers=1, agents=10, lo=200, hi=8000, new_lo=1, new_hi=40, pad=9, type="f16", fused=False, bf16=False),
        # a ragged prefill out of a fused bfloat16 projection
        dict(name="append_llama_prefill", kind="append", shape="llama", layers=4, agents=24, lo=0, hi=3500, new_lo=1, new_hi=700, pad=100, type="bf16", fused=True, bf16=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _row_bytes(shape):
    """Q4 bytes of one token's K and V rows in one layer."""
    _, hkv, dk, dv, alias = SHAPES[shape]
    width = dk if alias else dk + dv
    return hkv * (width // 2 + 4 * (width // GROUP))


def draw(rng):
    case = _draw(rng)
    most = {c["kind"]: max(work(d)["bytes"] for d in listed() if d["kind"] == c["kind"]) for c in listed()}
    while work(case)["bytes"] > most[case["kind"]]:       # no more than the largest listed case of its kind
        k = next(k for k in ("layers", "groups", "agents", "slack", "vocab") if case.get(k, 1) > 1)
        case[k] = max(1, case[k] * 3 // 4)
        if "new_lo" in case:
            case["new_lo"] = min(case["new_lo"], case["new_hi"])
    return case


def _draw(rng):
    kind = rng.choice(["select", "select", "select", "reorder", "reorder", "tables", "tables", "append"])
    if kind == "select":
        t = rng.choice(list(KINDS))
        vocab = _log_int(rng, 1000, 262144)
        beams = _log_int(rng, 1, 24)
        groups = max(1, min(_log_int(rng, 1, 96), 64 * 4 * 262144 // (vocab * beams * (2 if t == "f32" else 1))))
        return dict(kind=kind, groups=groups, beams=beams, ragged=rng.random() < 0.4, vocab=vocab, pad=rng.choice([0, 0, 1, rng.randint(1, 64)]),
                    out=max(1, min(64, rng.choice([beams, beams, 2 * beams, _log_int(rng, 1, 64)]))), type=t,
                    banned=rng.choice([0.0, 0.0, 0.5, 0.97]), finished=rng.choice([0.0, -1.0, 0.1, 0.4]))
    if kind == "reorder":
        shape, beams, bf16 = rng.choice(list(SHAPES)), _log_int(rng, 2, 20), rng.random() < 0.4
        layers = _log_int(rng, 1, 48)
        # no more bytes in the tails than the listed cases' largest, pools of a few GB
        most = 48 * 40 * 256 * _row_bytes("gemma")
        groups = max(1, min(_log_int(rng, 1, 24), most // (beams * layers * PAGE * _row_bytes(shape)), 400 // beams))
        blocks = max(1, min(12, int(6e9 / (layers * PAGE * _row_bytes(shape) * groups * (beams + 1)))))
        return dict(kind=kind, shape=shape, layers=layers, groups=groups, beams=beams, prompt=rng.randint(0, PAGE * blocks),
                    made=_log_int(rng, 1, PAGE * min(3, blocks)), bf16=bf16)
    if kind == "tables":
        agents, share = _log_int(rng, 1, 1000), rng.choice([1, 1, 4, 8])
        form = rng.choice(["step", "drafts", "admit"])
        lo, hi, grow_lo, grow_hi = 0, 0, 1, 1
        if form != "admit":
            hi = _log_int(rng, 1, 8000)
            lo = int(hi * rng.random())
        if form == "drafts":
            grow_hi = rng.randint(1, 16)
        if form == "admit":
            grow_hi = _log_int(rng, 1, max(1, min(20000, 400 * 1400 // agents)))
        return dict(kind=kind, agents=agents, share=share if form != "admit" else 1, lo=lo, hi=hi, grow_lo=min(grow_lo, grow_hi), grow_hi=grow_hi,
                    slack=_log_int(rng, 100, 20000), pad=rng.choice([0, rng.randint(1, 500)]))
    shape, agents = rng.choice(list(SHAPES)), _log_int(rng, 1, 60)
    _, hkv, dk, dv, alias = SHAPES[shape]
    width = hkv * (dk if alias else dk + dv)
    most = 4 * 24 * 350 * 2048  # values of the largest listed case
    layers = max(1, min(rng.randint(1, 6), most // (agents * width)))
    new_hi = _log_int(rng, 1, max(1, min(2000, 2 * most // (layers * agents * width))))
    hi = _log_int(rng, 1, 9000)
    return dict(kind=kind, shape=shape, layers=layers, agents=agents, lo=int(hi * rng.random()), hi=hi, new_lo=max(1, int(new_hi * rng.random())), new_hi=new_hi,
                pad=rng.choice([0, rng.randint(1, 60)]), type=rng.choice(["f16", "bf16"]), fused=rng.random() < 0.5, bf16=rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------ inputs

def _generator(*key):
    n = 0x2545F4914F6CDD1D
    for k in key:
        n = ((n ^ int(k)) * 0x9E3779B97F4A7C15 + 0x1234567) & ((1 << 62) - 1)
        n ^= n >> 29
    return torch.Generator(device="cuda").manual_seed(n)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _kind(bf16):
    return torch.bfloat16 if bf16 else torch.float16


def _of(case):
    """The case's own random numbers: what is the same for every seed."""
    return random.Random(" ".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _bounds(case):
    """First row of every group, and the number of rows."""
    rng, at = _of(case), [0]
    for _ in range(case["groups"]):
        at.append(at[-1] + (rng.randint(1, case["beams"]) if case["ragged"] else case["beams"]))
    return at


def _prepare_select(case, seed):
    bounds, rng, g = _bounds(case), random.Random(seed), _generator(seed, 1)
    rows, vocab = bounds[-1], case["vocab"]
    wide = torch.empty((rows, vocab + case["pad"]), dtype=KINDS[case["type"]], device="cuda")
    peak = torch.rand(rows, generator=g, device="cuda") * 3 + 1.5  # from nearly uniform rows to sharp ones
    for r in range(rows):
        x = torch.randn(vocab + case["pad"], generator=g, device="cuda") * peak[r]
        if case["banned"]:
            x = torch.where(torch.rand(x.shape, generator=g, device="cuda") < case["banned"], -math.inf, x)
        wide[r] = x
    scores, end = [], []
    for a, b in zip(bounds, bounds[1:]):
        for i in range(b - a):
            scores.append(-rng.random() * 12 if case["finished"] >= 0 else (0.0 if i == 0 else -math.inf))
            end.append(2 if case["finished"] > 0 and rng.random() < case["finished"] else -1)
    return dict(case=case, logits=wide[:, :vocab], scores=torch.tensor(scores, dtype=torch.float32, device="cuda"),
                end=_ints(end) if case["finished"] > 0 else None, bounds=_ints(bounds))


def _random_pool(seed, which, layers, pages, hkv, dim):
    """codes int32 [layers][pages][hkv][256][dim / 8], scale and bias bits int16 [..., dim / 64]."""
    g, shape = _generator(seed, 10 + which), (layers, pages, hkv, PAGE)
    return (torch.randint(-(1 << 31), 1 << 31, shape + (dim // 8,), generator=g, device="cuda", dtype=torch.int32),
            torch.randint(0x2C00, 0x3C00, shape + (dim // GROUP,), generator=g, device="cuda", dtype=torch.int16),
            torch.randint(-0x4400, -0x3C00, shape + (dim // GROUP,), generator=g, device="cuda", dtype=torch.int16))


def _listing(lens, heads, ids, width):
    """A block table for rows of these lengths (heads: blocks that row a begins with, else none), and how often each block is listed."""
    table, refs = np.full((len(lens), width), -1, np.int32), np.zeros(len(ids), np.int32)
    at = 0
    for a, n in enumerate(lens):
        mine = list(heads[a])
        while len(mine) < -(-n // PAGE):
            mine.append(ids[at])
            at += 1
        table[a, :len(mine)] = mine
        refs[mine] += 1
    return table, refs


def _prepare_reorder(case, seed):
    _, hkv, dk, dv, alias = SHAPES[case["shape"]]
    rng, layers, beams = _of(case), case["layers"], case["beams"]
    rows = case["groups"] * beams
    shared = case["prompt"] // PAGE                       # whole blocks of the prompt: the beams of a request list them together
    lens, parent = [], []
    for g in range(case["groups"]):
        made = max(1, case["made"] - rng.randint(0, min(30, case["made"] - 1)))
        lens += [case["prompt"] + made] * beams
        parent += [g * beams + min(rng.randrange(beams), rng.randrange(beams)) for _ in range(beams)]
    each = -(-max(lens) // PAGE)
    total = case["groups"] * shared + rows * (each - shared) + rows
    ids = list(range(total))
    random.Random(seed).shuffle(ids)
    heads = [ids[total - 1 - shared * (r // beams + 1):total - 1 - shared * (r // beams)] for r in range(rows)]
    table, refs = _listing(lens, heads, ids, each + 1)
    return dict(case=case, table=torch.from_numpy(table).cuda(), refs=torch.from_numpy(refs).cuda(), lens=_ints(lens), parent=_ints(parent),
                kpool=_random_pool(seed, 0, layers, total, hkv, dk), vpool=None if alias else _random_pool(seed, 1, layers, total, hkv, dv))


def _growth(case):
    """Old and new lengths, and the room for new tokens; the same for every seed."""
    rng = _of(case)
    old = [rng.randint(case["lo"], case["hi"]) for _ in range(case["agents"])]
    new = [n + rng.randint(case["grow_lo"], case["grow_hi"]) for n in old]
    return old, new, sum(new) - sum(old) + case["pad"]


def _prepare_tables(case, seed):
    old, new, room = _growth(case)
    total = sum(-(-n // PAGE) for n in new) + case["slack"]
    ids = list(range(total))
    random.Random(seed).shuffle(ids)
    heads = [[] for _ in old]
    if case["share"] > 1:                                 # rows in families that list the whole blocks of their shortest row together
        at = total
        for f in range(0, len(old), case["share"]):
            n = min(old[f:f + case["share"]]) // PAGE
            if n:
                heads[f:f + case["share"]] = [ids[at - n:at]] * len(old[f:f + case["share"]])
            at -= n
    table, refs = _listing(old, heads, ids, -(-max(new) // PAGE) + 1)
    refs[[i for i in ids if refs[i] == 0][:(case["slack"] + 1) // 2]] = 1  # blocks of agents that are not in this batch
    return dict(case=case, table=torch.from_numpy(table).cuda(), refs=torch.from_numpy(refs).cuda(), lens=_ints(old), old=_ints(old), new=_ints(new), room=room)


def _chunks(case):
    """Tokens cached before and appended now of every request; the same for every seed."""
    rng = _of(case)
    return [(rng.randint(case["lo"], case["hi"]), rng.randint(case["new_lo"], case["new_hi"])) for _ in range(case["agents"])]


def _prepare_append(case, seed):
    hq, hkv, dk, dv, alias = SHAPES[case["shape"]]
    layers, chunks, g = case["layers"], _chunks(case), _generator(seed, 1)
    need = [(n + m - 1) // PAGE - n // PAGE + 1 for n, m in chunks]
    ids = list(range(sum(need)))                          # the pages that the new tokens fall into
    random.Random(seed).shuffle(ids)
    slots, at = [], 0
    for (n, m), k in zip(chunks, need):
        slots += [ids[at + t // PAGE - n // PAGE] * PAGE + t % PAGE for t in range(n, n + m)]
        at += k
    slots += [-1] * case["pad"]                           # a batch of fixed size: what no request fills has no slot
    kind = KINDS[case["type"]]
    widths = [hkv * dk] + ([] if alias else [hkv * dv])
    if case["fused"]:
        x = torch.randn((layers, len(slots), hq * dk + sum(widths)), generator=g, device="cuda", dtype=kind)
        parts = list(x[..., hq * dk:].split(widths, -1))
    else:
        parts = [torch.randn((layers, len(slots), w), generator=g, device="cuda", dtype=kind) for w in widths]
    k, v = parts[0].unflatten(-1, (hkv, dk)), None if alias else parts[1].unflatten(-1, (hkv, dv))
    rng = random.Random(seed)
    for h in range(hkv):                                  # outlier channels
        k[..., h, rng.sample(range(dk), 4)] *= 8
    return dict(case=case, k=k, v=v, slot=_ints(slots), kpool=_random_pool(seed, 0, layers, len(ids), hkv, dk),
                vpool=None if alias else _random_pool(seed, 1, layers, len(ids), hkv, dv))


def prepare(case, seed):
    return {"select": _prepare_select, "reorder": _prepare_reorder, "tables": _prepare_tables, "append": _prepare_append}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------------------------ plain forms

def _select_plain(s):
    x, n, bounds = s["logits"].double(), s["case"]["out"], s["bounds"].long()
    top = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float64).min)  # a row that is banned whole: no continuation
    total = s["scores"].double()[:, None] + (x - top - (x - top).exp().sum(-1, keepdim=True).log())
    total = torch.where(x == -math.inf, -math.inf, total)
    if s["end"] is not None:                              # a finished row goes on with its end token, at its score
        is_end = torch.arange(x.shape[1], device=x.device) == s["end"][:, None]
        total = torch.where(s["end"][:, None] >= 0, torch.where(is_end, s["scores"].double()[:, None], -math.inf), total)
    beams = torch.arange(s["case"]["beams"], device=x.device)
    row = bounds[:-1, None] + beams
    inside = row < bounds[1:, None]
    total = torch.where(inside[..., None], total[row.clamp(max=x.shape[0] - 1)], -math.inf).flatten(1)
    best, at = total.sort(dim=-1, descending=True, stable=True)
    best, at = best[:, :n], at[:, :n]
    parent, token = bounds[:-1, None] + at // x.shape[1], at % x.shape[1]
    if best.shape[1] < n:
        best, parent, token = (torch.nn.functional.pad(t, (0, n - best.shape[1]), value=v) for t, v in ((best, -math.inf), (parent, -1), (token, -1)))
    none = best == -math.inf
    return [torch.where(none, -1, parent).int(), torch.where(none, -1, token).int(), best.float()]


def _counts(table, lens, refs):
    """How often the rows list each block."""
    listed = torch.arange(table.shape[1], device=table.device) * PAGE < lens[:, None]
    return torch.zeros_like(refs).index_add_(0, table[listed].long(), torch.ones_like(table[listed]))


def _reorder_plain(s):
    table, refs, lens, parent = s["table"], s["refs"], s["lens"], s["parent"].long()
    place, rows = torch.arange(table.shape[1], device=table.device), torch.arange(table.shape[0], device=table.device)
    new = lens[parent]
    held = place * PAGE < torch.maximum(lens, new)[:, None]
    table[:] = torch.where(place * PAGE < new[:, None], table[parent], torch.where(held, -1, table))
    lens[:] = new
    refs[:] = _counts(table, lens, refs)
    last = table[rows, (lens // PAGE).long().clamp(max=table.shape[1] - 1)].long().clamp(min=0)
    partial = lens % PAGE > 0
    first = torch.full_like(refs, len(rows)).scatter_reduce_(0, last[partial], rows[partial].int(), "amin")
    moves = partial & (first[last] != rows)
    src, used = last[moves], (lens % PAGE)[moves]
    dst = (refs == 0).nonzero()[:, 0][:len(src)]
    table[rows[moves], (lens // PAGE).long()[moves]] = dst.int()
    refs.index_add_(0, src, torch.full_like(used, -1))
    refs[dst] = 1
    pools = [t for p in (s["kpool"], s["vpool"]) if p is not None for t in p]
    copied = (torch.arange(PAGE, device=table.device) < used[:, None])[None, :, None, :, None]
    for t in pools:
        t[:, dst] = torch.where(copied, t[:, src], t[:, dst])
    return [table, refs, lens] + pools


def _resize_plain(table, refs, lens, new):
    place = torch.arange(table.shape[1], device=table.device) * PAGE
    gone = (place >= new[:, None]) & (place < lens[:, None])
    refs.index_add_(0, table[gone].long(), torch.full_like(table[gone], -1))
    table[gone] = -1
    more = (place >= lens[:, None]) & (place < new[:, None]) & (place >= (lens[:, None] + PAGE - 1) // PAGE * PAGE)
    free = (refs == 0).nonzero()[:, 0].int()[:int(more.sum())]
    table[more] = free
    refs[free.long()] = 1
    lens[:] = new


def _tables_plain(s):
    table, refs, lens, old, new = s["table"], s["refs"], s["lens"], s["old"], s["new"]
    _resize_plain(table, refs, lens, new)
    begin = torch.nn.functional.pad((new - old).cumsum(0), (1, 0)).int()
    t = torch.arange(s["room"], device=table.device)
    agent = (torch.searchsorted(begin, t.int(), right=True) - 1).clamp(max=len(old) - 1)
    position = old[agent] + (t - begin[agent])
    slot = table[agent, (position // PAGE).clamp(max=table.shape[1] - 1)] * PAGE + position % PAGE
    inside = t < begin[-1]
    slot, agent, position = (torch.where(inside, x, -1).int() for x in (slot, agent, position))
    _resize_plain(table, refs, lens, old)
    return [begin, slot, agent, position, table, refs, lens]


def _q4(x, bf16):
    """binary16 rows [..., width] to codes as float32, scales and biases as float32: the format's definition."""
    g = x.float().unflatten(-1, (-1, GROUP))
    low, high = g.amin(-1), g.amax(-1)
    scale = ((high - low) / torch.full_like(low, 15.0)).to(_kind(bf16)).float()  # by a tensor: a true division
    bias = low.to(_kind(bf16)).float()
    code = ((g - bias[..., None]) / torch.where(scale > 0, scale, 1.0)[..., None]).round().clamp(0, 15)
    return torch.where(scale[..., None] > 0, code, 0.0), scale, bias


def _values(pool, bf16):
    """The numbers that a pool's words stand for, in 32 bits."""
    codes, scale, bias = pool
    shift = torch.arange(0, 32, 4, device=codes.device, dtype=torch.int32)
    code = ((codes[..., None] >> shift) & 15).flatten(-2).unflatten(-1, (-1, GROUP)).float()
    return (code * scale.view(_kind(bf16)).float()[..., None] + bias.view(_kind(bf16)).float()[..., None]).flatten(-2)


def _append_plain(s):
    bf16, got = s["case"]["bf16"], []
    on = s["slot"] >= 0
    at = s["slot"][on].long()
    for pool, new in ((s["kpool"], s["k"]), (s["vpool"], s["v"])):
        if pool is None:
            continue
        code, scale, bias = _q4(new[:, on].half(), bf16)
        out = _values(pool, bf16).half()
        out[:, at // PAGE, :, at % PAGE] = (code * scale[..., None] + bias[..., None]).flatten(-2).half().transpose(0, 1)
        got.append(out)
    return got


# ------------------------------------------------------------------------------------------------ the framework's calls

def _handles(s):
    """What a program keeps between calls: spec and pools, tables, outputs and workspaces around the state's arrays."""
    if "b" not in s:
        from paper_2603_04428_amd import binding as b
        s["b"], case = b, s["case"]
        if case["kind"] in ("reorder", "append"):
            hq, hkv, dk, dv, alias = SHAPES[case["shape"]]
            s["spec"] = b.make_spec(case["layers"], hq, hkv, dk, dv, alias, param_format=b.PARAMS_BF16 if case["bf16"] else b.PARAMS_F16)
            s["pools"] = [None if p is None else b.Pool.of(*p) for p in (s["kpool"], s["vpool"])]
        if case["kind"] in ("reorder", "tables"):
            s["tables"] = b.BlockTables.of(s["table"], s["lens"], s["refs"])
            s["workspace"] = b.q4kv_tables_workspace(s["tables"])
        if case["kind"] == "tables":
            s["map"] = b.TokenMap(s["tables"], s["room"])
        if case["kind"] == "select":
            rows, vocab = s["logits"].shape
            s["workspace"] = b.q4kv_beam_select_workspace(s["logits"], case["out"])
            s["chosen"] = b.BeamChoice(case["groups"], case["out"])
    return s["b"]


def _select_own(s):
    b = _handles(s)
    chosen = b.q4kv_beam_select(s["logits"], s["scores"], s["bounds"], s["case"]["out"], end_token=s["end"], out=s["chosen"], workspace=s["workspace"])
    return [chosen.parent, chosen.token, chosen.score]


def _reorder_own(s):
    b = _handles(s)
    kpool, vpool = s["pools"]
    b.q4kv_beam_reorder(s["spec"], kpool, vpool, s["tables"], s["parent"], workspace=s["workspace"])
    return [s["table"], s["refs"], s["lens"]] + [t for p in (kpool, vpool) if p is not None for t in (p.codes, p.scale, p.bias)]


def _tables_own(s):
    b = _handles(s)
    b.q4kv_resize_tables(s["tables"], s["new"], out=s["map"], workspace=s["workspace"])
    b.q4kv_resize_tables(s["tables"], s["old"], workspace=s["workspace"])
    m = s["map"]
    return [m.begin, m.slot, m.agent, m.position, s["table"], s["refs"], s["lens"]]


def _append_own(s):
    b = _handles(s)
    kpool, vpool = s["pools"]
    b.q4kv_append_slots(s["spec"], kpool, vpool, s["k"], s["v"], s["slot"])
    return [b.q4kv_dequantize(p.codes, p.scale, p.bias, param_format=s["spec"].param_format) for p in (kpool, vpool) if p is not None]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"select": _select_own, "reorder": _reorder_own, "tables": _tables_own, "append": _append_own}[kind](state)
    return {"select": _select_plain, "reorder": _reorder_plain, "tables": _tables_plain, "append": _append_plain}[kind](state)


# ------------------------------------------------------------------------------------------------ work

def work(case):
    if case["kind"] == "select":
        rows, size = _bounds(case)[-1], 4 if case["type"] == "f32" else 2
        live = case["groups"] if case["finished"] < 0 else rows  # rows of score -inf have no continuation
        live *= 1 - max(0.0, case["finished"])
        return {"bytes": live * case["vocab"] * size + rows * 8 + 12 * case["groups"] * case["out"], "flops": 4 * live * case["vocab"]}
    if case["kind"] == "reorder":
        rng, beams, moved, rows = _of(case), case["beams"], 0, case["groups"] * case["beams"]
        for g in range(case["groups"]):
            made = max(1, case["made"] - rng.randint(0, min(30, case["made"] - 1)))
            parent = [min(rng.randrange(beams), rng.randrange(beams)) for _ in range(beams)]
            moved += (beams - len(set(parent))) * ((case["prompt"] + made) % PAGE)
        blocks = rows * -(-(case["prompt"] + case["made"]) // PAGE)
        return {"bytes": 2 * case["layers"] * moved * _row_bytes(case["shape"]) + rows * 12 + blocks * 12, "flops": 0}
    if case["kind"] == "tables":
        old, new, room = _growth(case)
        taken = sum(-(-n // PAGE) - -(-m // PAGE) for n, m in zip(new, old))
        blocks = sum(-(-n // PAGE) for n in new) + case["slack"]
        return {"bytes": 12 * room + 24 * case["agents"] + 4 * blocks + 16 * taken, "flops": 0}
    _, hkv, dk, dv, alias = SHAPES[case["shape"]]
    chunks, row = _chunks(case), _row_bytes(case["shape"])
    tokens, width = case["layers"] * sum(m for _, m in chunks), hkv * (dk if alias else dk + dv)
    places = case["layers"] * PAGE * sum((n + m - 1) // PAGE - n // PAGE + 1 for n, m in chunks)
    # rows in, cache rows out; the pages' rows of other tokens in, all of the pages' values out
    return {"bytes": tokens * (2 * width + row) + places * (row + 2 * width) - tokens * row + 4 * tokens, "flops": 4 * tokens * width}


# ------------------------------------------------------------------------------------------------ 64-bit results

def _exact_select(case, seed):
    s = _prepare_select(case, seed)
    bounds, n = _bounds(case), case["out"]
    scores, end = s["scores"].cpu().double().numpy(), None if s["end"] is None else s["end"].cpu().numpy()
    out = np.full((case["groups"], n), -np.inf)
    for g in range(case["groups"]):
        best = []
        for r in range(bounds[g], bounds[g + 1]):
            if end is not None and end[r] >= 0:
                best.append(np.array([scores[r]]))
                continue
            x = s["logits"][r].double()
            x = x[x > -math.inf]
            if x.numel() == 0 or scores[r] == -np.inf:
                continue
            top, _ = x.topk(min(n, x.numel()))
            best.append(scores[r] + (top - torch.logsumexp(x, 0)).cpu().numpy())
        if best:
            best = np.sort(np.concatenate(best))[::-1][:n]
            out[g, :len(best)] = best
    return [None, None, out]


def _numbers(words, scale, bias, bf16):
    """What Q4 rows stand for, in 64 bits (host arrays of words and parameter bits)."""
    codes = np.stack([(words.view(np.uint32) >> np.uint32(4 * i)) & np.uint32(15) for i in range(8)], -1)
    codes = codes.reshape(words.shape[:-1] + (-1, GROUP)).astype(np.float64)

    def wide(bits):
        if bf16:
            return (bits.view(np.uint16).astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
        return bits.view(np.float16).astype(np.float64)
    out = codes * wide(scale)[..., None] + wide(bias)[..., None]
    return out.reshape(out.shape[:-2] + (-1,))


def _to_param(x, bf16):
    """binary32 values to the nearest stored parameter, as binary64."""
    if bf16:
        u = x.astype(np.float32).view(np.uint32).astype(np.uint64)
        return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)).view(np.float32).astype(np.float64)
    return x.astype(np.float32).astype(np.float16).astype(np.float64)


def _requantized(x, bf16):
    """Rows of binary16 numbers (given as binary64) after a trip through Q4: subtraction and division are rounded to binary32."""
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    low, high = g.min(-1), g.max(-1)
    scale = _to_param((high - low).astype(np.float32) / np.float32(15), bf16)
    bias = _to_param(low, bf16)
    num = (g - bias[..., None]).astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.rint(num / scale.astype(np.float32)[..., None])
    code = np.where(scale[..., None] > 0, np.clip(code, 0, 15), 0).astype(np.float64)
    return (code * scale[..., None] + bias[..., None]).reshape(x.shape)


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    got = []
    for pool, new in ((s["kpool"], s["k"]), (s["vpool"], s["v"])):
        if pool is None:
            continue
        out = _numbers(*[t.cpu().numpy() for t in pool], case["bf16"])
        rows = _requantized(new.cpu().double().numpy().astype(np.float16).astype(np.float64), case["bf16"])
        for i, slot in enumerate(s["slot"].tolist()):
            if slot >= 0:
                out[:, slot // PAGE, :, slot % PAGE] = rows[:, i]
        got.append(out)
    return got


def exact(case, seed):
    if case["kind"] == "select":
        return _exact_select(case, seed)
    return _exact_append(case, seed) if case["kind"] == "append" else None
