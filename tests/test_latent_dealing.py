"""How latent attention deals units that are not cut: where there are shares enough, one a share at most.  The rule of csrc/attn_latent.hip (Share, Cut::whole, lead_of) in whole
numbers, with its constants from there."""
import os
import random
import re

import pytest

from launches import ROOT

SOURCE = open(os.path.join(ROOT, "paper_2603_10342_amd", "csrc", "attn_latent.hip")).read()
LEAD = int(re.search(r"kOnlyLead = (\d+)", SOURCE)[1])
TOKENS, MOST = (int(re.search(r"%s = (\d+)" % n, SOURCE)[1]) for n in ("kTokens", "kWholeTiles"))
LEAST = 8                                     # the most that a share has at least, in tiles


def units_of_shares(keys, shares, decode):
    """Units that every share takes, of units with so many keys: a unit goes to the share that has more of it."""
    unit = 1 if decode else TOKENS            # what costs are counted in, of a tile
    costs = [(-(-k // TOKENS) if decode else k) + LEAD * unit for k in keys]
    total = sum(costs)
    assert total + shares * (LEAST + 1) * unit < 1 << 31               # a decode's are 32-bit numbers
    per = max(-(-total // shares), min(total // len(costs), LEAST * unit))
    per = max(-(-per // unit) * unit, unit)
    takes, at = [0] * shares, 0
    for c in costs:
        w = at // per                         # cuts at w * per; one up to the middle leaves the unit to what follows
        while (w + 1) * per < at + c and 2 * ((w + 1) * per - at) <= c:
            w += 1
        takes[w] += 1
        at += c
    return takes


KEYS = TOKENS * MOST
ORDERS = {"short first": lambda n: [1] * (n // 2) + [KEYS] * (n - n // 2), "long first": lambda n: [KEYS] * (n // 2) + [1] * (n - n // 2),
          "rising": lambda n: [1 + i * (KEYS - 1) // n for i in range(n)], "all long": lambda n: [KEYS] * n, "all short": lambda n: [1] * n, "one long": lambda n: [1] * (n - 1) + [KEYS],
          "long but two": lambda n: [KEYS] * (n - 2) + [1] * 2, "drawn": lambda n: [random.Random(n).randint(1, KEYS) for _ in range(n)]}


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("decode", [True, False])
def test_no_share_has_two_units(order, decode):
    for shares in (256, 255, 224, 100, 32, 8):
        for n in {shares, shares - 1, shares - 2, shares * 3 // 4, shares // 2 + 1, 3}:
            takes = units_of_shares(ORDERS[order](n), shares, decode)
            assert sum(takes) == n and max(takes) == 1, (shares, n, takes)
