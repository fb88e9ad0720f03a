"""Calls of attention with masses, one or two for each way that a call is cut which takes many
units or columns: what they are, and the cut that the host code gives them (waves and LDS of
single tokens, tiles and splits of prompts)."""
from collections import namedtuple

import numpy as np

# n queries over L*B*Hkv units, the longest of `most` rows with room for 2 n more.
Path = namedtuple("Path", "name L B Hq Hkv n most cut")

TOKENS = [
    # Eight waves to a unit, all logits in LDS.
    Path("eight_held", 3, 11, 28, 4, 1, 4000, dict(waves=8, npmax=1, here=4032, ldr=0)),
    # The rest of a long unit's logits in the workspace.
    Path("eight_spilled", 3, 11, 28, 4, 1, 5500, dict(waves=8, npmax=1, here=4384, ldr=1120)),
    Path("eight_of_16", 2, 17, 64, 4, 1, 2500, dict(waves=8, npmax=1, here=1792, ldr=736)),
    Path("eight_drafts", 3, 11, 28, 4, 2, 4500, dict(waves=8, npmax=1, here=2048, ldr=2464)),
    # The same with four waves.
    Path("four_spilled", 4, 7, 28, 4, 1, 1500, dict(waves=4, npmax=1, here=1440, ldr=64)),
    Path("four_of_16", 2, 13, 64, 4, 1, 850, dict(waves=4, npmax=1, here=576, ldr=288)),
    Path("four_drafts", 4, 7, 28, 4, 2, 980, dict(waves=4, npmax=1, here=672, ldr=320)),
]
PROMPTS = [
    # Whole tiles of 256 columns, masses of several parts and of one.
    Path("whole_256", 1, 4, 28, 4, 330, 700, dict(qcols=256, nqt=10, ns=1, csplit=4)),
    Path("whole_256_masses_too", 4, 9, 28, 4, 40, 600, dict(qcols=256, nqt=2, ns=1, csplit=1)),
    # Whole tiles of 128 columns over more rows than a split leaves together.
    Path("whole_128", 6, 11, 28, 4, 17, 700, dict(qcols=128, nqt=1, ns=1, csplit=1)),
]
SHORT = [0, 1, 31, 32, 33, 63, 64, 65, 127, 129, 200, 511]


def sizes(p):
    """(lens, caps) of the units: most of them short, four near the longest."""
    rng = np.random.default_rng(p.most)
    units = p.L * p.B * p.Hkv
    lens = [int(x) for x in rng.choice(SHORT, units)]
    caps = [x + 2 * p.n + int(rng.integers(0, 3)) for x in lens]
    for u, x in ((1, p.most), (units // 3, p.most - 33), (units // 2, p.most * 2 // 3), (units - 1, p.most - 64)):
        lens[u], caps[u] = x, x + 2 * p.n
    return lens, caps
