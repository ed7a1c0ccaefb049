"""q4kv_beam_select on rows whose sums of exponentials change their reference on the way, at logits of any size.

The bound is the header's.  A wave sums terms 2^(x c - m) over its part of a row, m being the reference r times c rounded once; what m is
off by is taken out in binary64, at the end and where the reference moves.  With d = x - r, r the reference when x was summed, the
exponent's rounding puts a term off by |d| 2^-24; the constant c, binary32's log2 e or the number above it, by up to 1.16 |d'| 2^-24, d'
counted from the last reference; the exponential by 2^-23; sums of twelve such by 12 * 2^-24.  No d or d' is above 8: there the reference
moves.  Below the reference the mean of -d over n terms weighted with e^d, of which one is e^0, is at most ln(n) (the weights' entropy,
less the logarithm of their sum).  So both means of |d| are at most ln(vocab) + 8, and with 2^-22 for what follows the logarithm is
within (1.08 (ln(vocab) + 8) + 7 + 2) 2^-23, which is below (1.1 ln(vocab) + 18) 2^-23."""
import numpy as np
import pytest
import torch

from tests.test_gpu_beam_select import KINDS, check

pytestmark = pytest.mark.gpu

STEP = 2048                                                # elements that a wave looks at together
SIZES = {"f16": [1.0, 30.0, 100.0, 1000.0, 10000.0, 60000.0], "bf16": [1.0, 30.0, 100.0, 1000.0, 500000.0],
         "f32": [1.0, 30.0, 100.0, 1000.0, 5000.0, 10000.0, 500000.0, 5000000.0]}


def above(x, kind):
    """The next number of the type that is at least 1 / 1024 above x."""
    t = torch.tensor(x, dtype=torch.float64)
    up = t.to(KINDS[kind])
    while up.double() < t + 2.0 ** -10:
        up = torch.nextafter(up.float(), torch.tensor(np.inf)).to(KINDS[kind]) if kind == "f32" else (up.view(torch.int16) + (1 if up > 0 else -1)).view(up.dtype)
    return up.item()


def row(kind, base, steps, form):
    """Steps of a row.  moves: all of the first step at base, one element 8 and a little above in the second, the rest below;
    plateau: a step 8 above the first, as far as the reference does not move, and one element that moves it; stairs: every step
    more than 8 above the one in front of it, half of it just under the limit of the next."""
    x = torch.full((steps * STEP,), base - 20.0, dtype=torch.float64)
    if form == "moves":
        x[:STEP] = base
        x[STEP:] = base - 3
        x[STEP + 977] = above(base + 8.6, kind)
    elif form == "plateau":
        x[:STEP] = base
        x[STEP:2 * STEP] = base + 8
        x[2 * STEP + 904] = above(base + 8.0, kind)
    else:
        for k in range(steps):
            x[k * STEP] = base if k == 0 else above(x[(k - 1) * STEP].item() + 8.0, kind)
            top = x[k * STEP].item()
            x[k * STEP + 1:(k + 1) * STEP] = top - 1
            if k:
                x[(k - 1) * STEP + STEP // 2:k * STEP] = torch.tensor(top - 8.001).to(KINDS[kind]).item() if kind == "f32" else x[(k - 1) * STEP].item()
    return x.to(KINDS[kind])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ["moves", "plateau", "stairs"])
def test_the_reference_moves(kind, form):
    """Rows at several sizes, side by side in one group and each in its own; 20 and 64 out: spans of two and of four steps."""
    for sign in (1.0, -1.0):
        rows = torch.stack([row(kind, sign * n, 4, form) for n in SIZES[kind]])
        n = len(rows)
        for num_out in (20, 64):
            check(rows, [-1.0] * n, [0, n], num_out)
            check(rows, [-1.0] * n, list(range(n + 1)), num_out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", ["moves", "plateau", "stairs"])
def test_the_reference_moves_in_a_span_of_eight_steps(kind, form):
    """So long are spans where there are many rows; all but a few are dead."""
    live = SIZES[kind][2:]
    rows = torch.zeros((2048, 8 * STEP), dtype=KINDS[kind])
    score = [-float("inf")] * 2048
    for i, n in enumerate(live):
        rows[300 * i + 7], score[300 * i + 7] = row(kind, n, 8, form), -1.0
    check(rows, score, [0, 2048], 8)


@pytest.mark.parametrize("kind", KINDS)
def test_the_reference_moves_behind_a_tail(kind):
    """What does not fill a load at a span's end is summed with its first step: such elements near the top, and a later step above them."""
    for size in SIZES[kind][1:5]:
        x = row(kind, size, 4, "plateau")
        for extra in (1, 3, 5, 7):
            tail = torch.full((extra,), size + 7.9, dtype=torch.float64).to(KINDS[kind])
            rows = torch.cat([x, tail])[None].repeat(2, 1)
            check(rows, [-1.0, -1.5], [0, 2], 64)


@pytest.mark.parametrize("kind", KINDS)
def test_the_reference_moves_where_values_are_replaced(kind):
    """The careful second reading: NaN and banned tokens among them, and sizes beyond 700,000."""
    sizes = SIZES[kind] + ([1e6, 1e30] if kind != "f16" else [])
    for form in ("moves", "plateau", "stairs"):
        rows = torch.stack([row(kind, n, 4, form) for n in sizes])
        rows[:, 100::STEP] = float("nan")
        rows[:, 101::STEP] = -float("inf")
        check(rows, [-1.0] * len(rows), list(range(len(rows) + 1)), 64)


def test_rows_are_ranked_by_their_own_sums():
    """Two rows of one group whose totals are 2^-15 apart: what a moved reference is off by may not exchange them."""
    a = row("f32", 500000.0, 4, "plateau")
    b = a - 490000.0                                       # exact: the same differences, another size
    for lead in (0, 1):
        score = [-1.0, -1.0]
        score[lead] += 2.0 ** -15
        out = check(torch.stack([a, b]), score, [0, 2], 64)
        assert out.parent[0, 0].item() == lead
