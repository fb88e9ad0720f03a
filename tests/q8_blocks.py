"""Attention over 8-bit caches in which every block counts: small queries, so that
all rows weigh about the same, and in every block of 64 rows one channel of the
values that is loud, its sign at random.  A block that is lost or taken twice then
moves an output by about its share of the rows times the loud value, far more than
the roundings may."""
import numpy as np

from tests import q8_ref as ref

LOUD = 4.0


class Case:
    """n queries (counts per sequence) of G heads per kv head over units of these
    lengths; `cut`: whether units or tiles are cut along their rows."""

    def __init__(self, name, B, Hkv, G, d, lens, n, cut, L=1, counts=None, causal=True, most=None, sample=None):
        self.name, self.L, self.B, self.Hkv, self.G, self.d, self.n, self.cut = name, L, B, Hkv, G, d, n, cut
        self.lens, self.causal, self.most = list(lens), causal, most
        self.counts = [n] * B if counts is None else list(counts)
        self.ragged = counts is not None
        self.sample = sorted({0, n // 3, n - 1}) if sample is None else sample
        assert len(self.lens) == L * B * Hkv and len(self.counts) == B


def _spread(seed, n, lo, hi):
    """Lengths over their logarithm, the open blocks empty or of at least 20 rows."""
    x = np.exp(np.random.default_rng(seed).uniform(np.log(lo), np.log(hi), n)).astype(int)
    return [int(v - v % 64 if v % 64 < 20 else v) for v in np.maximum(x, 64)]


CASES = [
    Case("pieces", 2, 2, 7, 128, [20011, 84, 6400, 9980], 1, True),
    Case("pieces_d64", 1, 2, 16, 64, [8063, 5000], 1, True),
    Case("pieces_of_drafts", 2, 1, 8, 64, [20011, 6420], 2, True),
    Case("whole_units", 40, 4, 7, 128, _spread(1, 160, 64, 1500), 1, False),
    Case("bounded", 1, 4, 4, 128, [9000, 4000, 2100, 700], 1, True, most=3200),
    Case("draft", 2, 2, 7, 128, [20011, 84, 6400, 9980], 9, True),
    Case("shares", 1, 2, 8, 128, [9020, 5000], 40, True),
    Case("shares_not_causal", 1, 2, 8, 128, [9020, 5000], 40, True, causal=False),
    Case("shares_counts", 5, 1, 8, 128, [9020, 5000, 84, 3000, 6464], 40, True, counts=[40, 0, 17, 3, 40]),
    Case("shares_wide_groups", 3, 1, 16, 64, [8980, 4600, 6400], 20, True, counts=[20, 11, 20]),
    Case("shares_unlike", 40, 2, 4, 64, _spread(2, 80, 64, 4000), 20, True),
    Case("shares_bounded", 1, 2, 8, 64, [9020, 5000], 40, True, most=4000, causal=False),
    # Whole tiles of 256 columns, also over so few blocks that the two phases hardly meet,
    # and of 128.
    Case("whole_tiles", 2, 8, 8, 128, [84, 64, 128, 150, 192, 225, 256, 300, 320, 1000, 1500, 2000, 2500, 2600, 700, 2560],
         264, False, sample=[0, 31, 32, 100, 131, 199, 200, 263]),
    Case("whole_tiles_d64", 2, 8, 8, 64, _spread(3, 16, 64, 2500), 264, False, sample=[0, 31, 100, 199, 263]),
    Case("whole_small_tiles", 130, 2, 4, 128, _spread(4, 260, 64, 700), 20, False),
    Case("whole_tiles_not_causal", 2, 8, 8, 128, _spread(5, 16, 64, 2500), 264, False, causal=False, sample=[0, 131, 263]),
]


def data(case):
    """(K, V per unit, q [L, B, n, Hq, d]) in bf16 values."""
    rng = np.random.default_rng(sum(map(ord, case.name)))
    d, K, V = case.d, [], []
    for u, n in enumerate(case.lens):
        K.append(ref.bf16(rng.standard_normal((n, d))))
        v = 0.25 * rng.standard_normal((n, d))
        for j in range((n + 63) // 64):
            v[64 * j:64 * j + 64, (7 * j + 3 * u) % d] += rng.choice((-LOUD, LOUD))
        V.append(ref.bf16(v))
    q = ref.bf16(0.3 * rng.standard_normal((case.L, case.B, case.n, case.G * case.Hkv, d)))
    return K, V, q


def expected(case, K, V, q, u, fp32, blocks=False):
    """The sampled rows of unit u over K, V as they read back: a list of (query, outputs
    [G, d], tolerance [G, d]) and, with `blocks`, what each block's loss and doubling
    would make of them, [2, blocks, G, d], and the rows of each block that are seen.

    The tolerance: q8_ref's, whose terms are all relative to a row's weight, so that
    they are relative to sum p |V| in each channel; with bf16 outputs the weights' rounding
    to fp16 (2^-11 of them, all far from its subnormals here) and the output's (2^-8 of
    itself) as well."""
    l, b, g = u // (case.B * case.Hkv), u // case.Hkv % case.B, u % case.Hkv
    scale, c, n = case.d ** -0.5, min(max(case.counts[b], 0), case.n), len(K)
    rows = []
    for i in case.sample:
        if i >= c:
            continue
        end = max(min(n - c + i + 1 if case.causal else n, n if case.most is None else case.most, n), 0)
        x = q[l, b, i, g * case.G:(g + 1) * case.G].astype(np.float64)
        if end == 0:
            rows.append((i, np.zeros((case.G, case.d)), np.zeros((case.G, case.d)), None, None))
            continue
        s = x @ K[:end].T * scale
        p = np.exp(s - s.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        want, size = p @ V[:end], p @ np.abs(V[:end])
        reach = (np.abs(x) @ np.abs(K[:end]).T).max() * scale
        tol = ref.tolerance(end, case.d, float(reach), 1.0, True) * size
        if not fp32:
            tol = tol + 2.0 ** -11 * size + 2.0 ** -8 * np.abs(want)
        moved = seen = None
        if blocks:
            nb = (end + 63) // 64
            pad = lambda a, k: np.concatenate((a, np.zeros(a.shape[:k] + (nb * 64 - end,) + a.shape[k + 1:])), axis=k)  # noqa: E731
            pb = pad(p, 1).reshape(case.G, nb, 64).transpose(1, 0, 2)
            part = pb @ pad(V[:end], 0).reshape(nb, 64, case.d)  # [nb, G, d]
            w = pb.sum(axis=2)[..., None]
            with np.errstate(divide="ignore", invalid="ignore"):
                moved = np.stack([np.nan_to_num((want - part) / (1 - w), posinf=0.0, neginf=0.0) if nb > 1 else 0 * part,
                                  (want + part) / (1 + w) if nb > 1 else want + 0 * part])
            seen = np.minimum(end - 64 * np.arange(nb), 64)
        rows.append((i, want, tol, moved, seen))
    return rows
