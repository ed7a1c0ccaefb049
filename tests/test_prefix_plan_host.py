"""How the tiles of a shared-prefix call are dealt out (csrc/prefix_plan.h), for 256 workgroups of four waves: every place in the
plan stays below 2^31, and the workers' ranges hold all that the units count for."""
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def spread(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "prefix_plan_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-Wall", "-Werror", "-Wno-unknown-pragmas", "-o", exe,
                    os.path.join(HERE, "host_c", "prefix_plan_check.cpp")], check=True)

    def ask(*units):
        out = subprocess.run([exe, "256", *("%d:%d" % u for u in units)], capture_output=True, text=True, check=True).stdout
        return [int(x) for x in out.split()]
    return ask


CALLS = {
    "one tile": [(1, 1)],
    "two agents behind 1,024": [(8, 16), (16, 2)],
    "ten behind 8,192": [(8, 128), (80, 7)],
    "32 behind 16,384, two layers": [(64, 256), (512, 12)],
    "twelve layers": [(96, 128), (960, 5)],
    "a unit for each wave, and one more": [(1025, 40)],
    "as many long units as waves": [(1024, 2 ** 31 // 1024 - 64)],
    "a few units, 2^31 tiles": [(3, 2 ** 31 // 3 - 40000)],
    "units that would be counted as twice their tiles": [(560, 3400000)],
    "long ones beside short ones": [(500, 4000000), (400, 1)],
    "half of all that there may be": [(900, 1150000)],
    "all that there may be": [(1, 0x7fff0000)],
}


@pytest.mark.parametrize("name", list(CALLS))
def test_places_stay_below_2_to_the_31(spread, name):
    units = CALLS[name]
    total = sum(n * t for n, t in units)
    assert total <= 0x7fff0000
    per, round_, solo, counted = spread(*units)
    assert total <= counted <= MOST
    assert counted <= per * (1024 if solo else 256) and per >= (2 if solo else 4) and round_ in (1, per)
    slots = max(-(-t // round_) * round_ // per + 2 for _, t in units)       # records of a unit
    assert slots <= max(max(t for _, t in units) // (2 if solo else 4), 1024 if solo else 256) + 2


def test_every_count_of_long_units(spread):
    for n in list(range(1, 1030, 13)) + [511, 512, 513, 1023, 1024, 1025]:
        for top in (0x7fff0000, 2 ** 30 + 12345, 2 ** 29):
            per, round_, solo, counted = spread((n, top // n))
            assert counted <= MOST and counted <= per * (1024 if solo else 256)


def test_records_of_a_row_stay_in_what_is_reserved(spread):
    """The records that a row's prefix and own tokens leave together, for random calls laid out as the kernel does: no more than
    min(tiles / 2, 1024 / pairs) or min(tiles / 4, 256 / pairs) of a row's longest, whichever is more, and four."""
    rng = random.Random(5)
    closest = 99
    for _ in range(400):
        pairs = rng.choice([1, 1, 2, 3, 8, 16, 40, 96])                              # (layer, KV head)
        top = rng.choice([1, 3, 17, 64, 130, 257, 600])                               # tiles of max_seq_len
        units = []                                                                    # of a pair: (tiles, rows that it serves), prefixes first
        agents = []
        for g in range(rng.randint(1, 4)):
            shared, crowd = rng.choice([0, rng.randint(0, top)]), rng.choice([1, 2, 5, 20])
            first = len(agents)
            agents += [(shared if crowd > 1 else 0, rng.choice([top, 0, rng.randint(0, top)])) for _ in range(crowd)]
            if crowd > 1 and shared:
                for r in range(0, crowd, 8):                                          # eight agents' rows a tile
                    units.append((shared, range(first + r, min(first + r + 8, first + crowd))))
        units += [(max(0, n - shared), [a]) for a, (shared, n) in enumerate(agents)]
        if not any(t for t, _ in units):
            continue
        per, round_, solo, _ = spread(*[(pairs, t) for t, _ in units if t])
        at = 0
        for _ in range(pairs):
            records = [0] * len(agents)
            for t, serves in units:
                counted = -(-t // round_) * round_
                for a in serves if t else ():
                    records[a] += (at + counted - 1) // per - at // per + 1
                at += counted
            slots = max(min(top // 2, 1024 // pairs), min(top // 4, 256 // pairs)) + 4
            assert max(records) <= slots
            closest = min(closest, slots - max(records))
    assert closest <= 3                                                               # the calls come near
