"""How the blocks of decode attention share the requests out (csrc/any4_attn_decode.hip), on the CPU: the kernel's integer formulas
again, for every block, against what they are to give."""
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2507_04610_amd", "csrc", "any4_attn_decode.hip")


def constant(name):
    with open(SOURCE) as f:
        return int(re.search(rf"constexpr int {name} = (\d+);", f.read()).group(1))


STEP, WHOLE = constant("kStep"), constant("kWholeUnits")


def shares(lengths, capacity, waves, groups, grid):
    """[(block, request, group, from, to, units, pieces, first block, place)], as the kernel goes through them"""
    unit = STEP * waves
    units_of = [max((min(max(n, 0), capacity) + unit - 1) // unit, 1) for n in lengths]
    begins = [0]
    for u in units_of:
        begins.append(begins[-1] + u)
    total, requests = begins[-1] * groups, len(lengths)
    blocks = min(grid, requests * groups if total < WHOLE * requests * groups else total)
    each, longer = total // blocks, total % blocks

    def block_of(x):
        return x // (each + 1) if x < longer * (each + 1) else longer + (x - longer * (each + 1)) // each
    found = []
    for block in range(blocks):
        at = block * each + min(block, longer)
        end = at + each + (1 if block < longer else 0)
        lo, hi, y = 0, requests - 1, at // groups
        while lo < hi:
            mid = (lo + hi + 1) >> 1
            lo, hi = (mid, hi) if begins[mid] <= y else (lo, mid - 1)
        request = lo
        # the search over the lanes of up to 64 requests gives the same one
        assert request == max(r for r in range(requests) if begins[r] <= y)
        while at < end:
            units = units_of[request]
            group = (at - begins[request] * groups) // units
            while group < groups and at < end:
                first = begins[request] * groups + group * units
                a, b = at - first, min(units, end - first)
                at = first + b
                first_block = block_of(first)
                found.append((block, request, group, a, b, units, block_of(first + units - 1) - first_block + 1, first_block, 0 if a > 0 else 1))
                group += 1
            request += 1
    return found, units_of, blocks


def check(lengths, capacity, waves, groups, grid):
    found, units_of, blocks = shares(lengths, capacity, waves, groups, grid)
    covered, places, pieces = {}, set(), {}
    for block, request, group, a, b, units, count, first_block, place in found:
        assert 0 <= a < b <= units == units_of[request] and block < blocks <= grid
        covered.setdefault((request, group), []).append((a, b))
        if a > 0 or b < units:                                   # a cut group: its result has a place of its own
            assert (block, place) not in places
            places.add((block, place))
            pieces.setdefault((request, group), []).append((block, place, count, first_block))
        else:
            assert count == 1
    for key, parts in covered.items():
        assert [a for a, _ in parts] == [0] + [b for _, b in parts[:-1]] and parts[-1][1] == units_of[key[0]]
    assert len(covered) == len(lengths) * groups
    for parts in pieces.values():                                # where the one that joins looks for piece w
        assert len(parts) == parts[0][2] <= grid
        assert [(b, p) for b, p, _, _ in parts] == [(parts[0][3] + w, 1 if w == 0 else 0) for w in range(len(parts))]
    loads = {}
    for block, _, _, a, b, *_ in found:
        loads[block] = loads.get(block, 0) + b - a
    assert max(loads.values()) - min(loads.values()) <= 1


@pytest.mark.parametrize("waves,grid", [(8, 256), (4, 512), (4, 768), (8, 1), (4, 3)])
@pytest.mark.parametrize("lengths,groups", [([0], 1), ([1], 8), ([333], 8), ([131071], 8), ([9001, 0, 5, 4096, 2049], 1), ([0] * 70, 2),
                                            (list(range(0, 4096, 130)), 8), ([1] * 31 + [100000], 3), ([8192] * 64, 8), ([2047] * 2048, 1)])
def test_every_unit_once(waves, grid, lengths, groups):
    check(lengths, 1 << 20, waves, groups, grid)


def test_random_calls():
    rng = random.Random(5)
    for _ in range(300):
        lengths = [rng.choice((0, 1, rng.randrange(300), rng.randrange(5000))) for _ in range(rng.choice((1, 2, 7, 33, 64, 65, 200)))]
        check(lengths, rng.choice((256, 4096, 1 << 20)), rng.choice((4, 8)), rng.choice((1, 2, 8, 24)), rng.choice((1, 5, 64, 256, 512, 768)))
