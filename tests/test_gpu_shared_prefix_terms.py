"""How many bits the weights of the values keep in q4kv_shared_prefix_attention: p s goes into the products in two binary16
terms.  Queries of one element make scores that are a single product, so that what is seen is the value side; a few tokens whose
values cancel make outputs small beside what is summed."""
import numpy as np
import pytest
import torch

import oracle
from paper_2603_04428_amd import binding as b
from tests.gpu_util import DEV
from tests.util import unpack_codes

HEADS = {"128": (8, 2, 128, 128), "256": (4, 2, 256, 256), "192": (3, 3, 192, 128), "64": (8, 1, 64, 64)}
PREFIX, OWN = 64, (1, 2, 5)          # agents 0 to 2 share 64 tokens (and keep a copy each); agents 3 to 5 have 2, 3 and 4 of their own
LENS = [PREFIX + n for n in OWN] + [2, 3, 4]
# of the values' groups: ordinary; the last with which weights reach 2^15 and the next in binary16 and in bfloat16; the same for 2^7;
# wide
SCALES = [0.3, 1.900390625, 1.9013671875, 1.90625, 252.0, 252.125, 254.0, 4000.0]


def build(heads, scale, fmt, seed):
    hq, hkv, dk, dv = heads
    rng, A = np.random.default_rng(seed), len(LENS)
    spec = oracle.make_spec(1, hq, hkv, dk, dv, param_format=fmt)
    kp, vp = oracle.Pool(spec, dk, A), oracle.Pool(spec, dv, A)
    table = np.arange(A, dtype=np.int32)[:, None]
    k = rng.standard_normal((1, A, max(LENS), hkv, dk)).astype(np.float16)
    v = rng.uniform(-7.5, 7.5, (1, A, max(LENS), hkv, dv // 64, 64)) * scale
    v[..., 0], v[..., 1] = -7.5 * scale, 7.5 * scale
    v = v.reshape(1, A, max(LENS), hkv, dv).astype(np.float16)
    for x in (k, v):
        x[:, :3, :PREFIX] = x[:, :1, :PREFIX]
    for a, n in enumerate(LENS):
        oracle.append(spec, kp, vp, np.ascontiguousarray(k[:, a:a + 1, :n]), np.ascontiguousarray(v[:, a:a + 1, :n]), table[a:a + 1], np.zeros(1, np.int32))
    q = np.zeros((1, A, 1, hq, dk), np.float16)
    for a in range(A):
        for h in range(hq):
            q[0, a, 0, h, rng.integers(dk)] = 0.5 * np.sqrt(dk)
    return spec, kp, vp, q, table


def wide(bits, fmt):
    bits = bits.view(np.uint16)
    return ((bits.astype(np.uint32) << 16).view(np.float32) if fmt else bits.view(np.float16)).astype(np.float64)


def limit(want, vp, fmt):
    """Half a step of the output, 2^-11 of it; of a group's scale s: 23 * 2^-19 for what matrix instructions cut off of the sums
    of 15 p s and 8 p s at most, 15 * 2^-19 for probabilities good to 2^-20 on both sides of the quotient, 8 * 2^-22 for two terms of
    p s, below 2^-13.5 together; 2^-20 of the middle b + 8 s for the two terms of p, their sum and the quotient."""
    s, bias = wide(vp.scale, fmt), wide(vp.bias, fmt)
    return 2.0 ** -11 * np.abs(want) + 2.0 ** -13.5 * s.max() + 2.0 ** -20 * np.abs(bias + 8 * s).max() + 2.0 ** -25


def want_of(spec, kp, vp, q, table):
    return oracle.attention(spec, kp, vp, q, table, LENS, 1 / np.sqrt(spec.k_dim), return_f64=True)[1]


def emulate(spec, kp, vp, q, table, fmt, terms):
    """The value side with p s in `terms` binary16 terms, everything else in binary64."""
    out = np.zeros(q.shape[:4] + (spec.v_dim,))
    rep = spec.num_q_heads // spec.num_kv_heads
    for a, n in enumerate(LENS):
        for h in range(spec.num_q_heads):
            g = h // rep
            s, bias = (np.repeat(wide(x[0, a, g, :n], fmt), 64, -1) for x in (vp.scale, vp.bias))
            c = unpack_codes(vp.codes[0, a, g, :n]).astype(np.float64)
            p = oracle.attention_probs(spec, kp, vp, 0, table[a], g, q[0, a, 0, h], n, 1 / np.sqrt(spec.k_dim))[0]
            p = p / p.max() * (4096.0 if s.max() <= 1.9004 else 16.0 if s.max() <= 252 else 1.0)
            ps = (p[:, None] * s).astype(np.float16).astype(np.float64)
            if terms == 2:
                ps += (p[:, None] * s - ps).astype(np.float16)
            out[0, a, 0, h] = (((c - 8) * ps).sum(0) + (p[:, None] * (bias + 8 * s)).sum(0)) / p.sum()
    return out.astype(np.float16).astype(np.float64)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("heads", HEADS.values(), ids=HEADS.keys())
def test_one_term_would_be_seen(heads, scale, fmt):
    made = build(heads, scale, fmt, 3)
    want = want_of(*made)
    lim = limit(want, made[2], fmt)
    assert np.all(np.abs(emulate(*made, fmt, 2) - want) <= lim)
    over = np.abs(emulate(*made, fmt, 1) - want) / lim
    assert np.mean(over > 1) > 0.02 and over.max() > 2


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("heads", HEADS.values(), ids=HEADS.keys())
def test_weights_keep_two_terms(heads, scale, fmt):
    made = build(heads, scale, fmt, 3)
    ospec, okp, ovp, q, table = made
    spec = b.make_spec(1, *heads, param_format=fmt)
    kp, vp = b.Pool(spec, heads[2], len(LENS), DEV), b.Pool(spec, heads[3], len(LENS), DEV)
    for g, o in ((kp, okp), (vp, ovp)):
        for name, kind in (("codes", np.int32), ("scale", np.int16), ("bias", np.int16)):
            getattr(g, name).copy_(torch.from_numpy(getattr(o, name).view(kind)))
    dev = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    got = b.q4kv_shared_prefix_attention(spec, kp, vp, torch.from_numpy(q).to(DEV), dev(table), dev(LENS), dev([0, 3]), dev([PREFIX]),
                                         max(LENS), 1 / np.sqrt(heads[2])).cpu().numpy().astype(np.float64)
    want = want_of(*made)
    over = np.abs(got - want) / limit(want, ovp, fmt)
    assert over.max() <= 1, over.max()
