"""Attention with masses on the ways through its kernels that take many units or columns
(tests/mass_paths.py), against 64 bits; tolerances are derived in tests/mass_ref.py."""
import numpy as np
import pytest

from tests import mass_paths as mp
from tests.test_gpu_mass_attend import _bf16, dev  # noqa: F401
from tests.test_gpu_mass_finite import Finite

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _pair(p, dev, d, seed=43):  # noqa: F811
    lens, caps = mp.sizes(p)
    return Finite(seed, dev, p.L, p.B, p.Hq, p.Hkv, d, lens, caps)


@pytest.mark.parametrize("p", mp.TOKENS + mp.PROMPTS, ids=lambda p: p.name)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fp32", [True, False])
def test_parity(dev, p, d, fp32):  # noqa: F811
    """A call that appends, one with counts and decay, and one over rows that are there."""
    x = _pair(p, dev, d)
    x.attend(*x.inputs(p.n), fp32=fp32)
    count = [int(c) for c in np.random.default_rng(p.n).integers(0, p.n + 1, p.B)]
    count[0], count[p.B - 1] = p.n, 0
    x.attend(*x.inputs(p.n), fp32=fp32, count=count, decay=0.5)
    x.attend(x.inputs(p.n)[0], fp32=fp32, decay=0.9, max_rows=max(x.c.cap.tolist()) - 1)


@pytest.mark.parametrize("p", [p for p in mp.TOKENS + mp.PROMPTS if p.n > 1], ids=lambda p: p.name)
@pytest.mark.parametrize("fp32", [True, False])
def test_rows_without_finite_values(dev, p, fp32):  # noqa: F811
    """A value that is not finite, in a new row and in an old one of every unit of two heads:
    it reaches the queries that see the row in its channel, and changes nothing else."""
    d, G, r = 64, p.Hq // p.Hkv, p.n // 2
    clean, x = _pair(p, dev, d), _pair(p, dev, d)
    q, k, v = (_bf16(t, dev) for t in clean.inputs(p.n))
    typ = torch.float32 if fp32 else torch.bfloat16
    want, out = (torch.zeros(q.shape, dtype=typ, device=dev) for _ in range(2))
    clean.c.attend(q, want, d ** -0.5, k=k, v=v)
    assert torch.isfinite(want).all()
    v[:, :, r, 0, 3] = float("inf")
    v[:, :, r, 1, 9] = float("nan")
    old = torch.zeros(q.shape, dtype=torch.bool, device=dev)
    for u, (unit, o) in enumerate(zip(x.units, x.off)):
        if u % p.Hkv == 2 and len(unit.K):  # its last row, which every query sees
            x.c.v_pool[o + len(unit.K) - 1, 5] = float("-inf")
            old[u // (p.B * p.Hkv), u // p.Hkv % p.B, :, 2 * G:3 * G, 5] = True
    x.c.attend(q, out, d ** -0.5, k=k, v=v)
    bad = torch.isfinite(out).logical_not()
    old[:, :, r:, :G, 3] = True
    old[:, :, r:, G:2 * G, 9] = True
    assert torch.equal(bad, old)
    assert torch.equal(out[~bad], want[~bad])
    assert torch.equal(x.c.mass, clean.c.mass)  # weights are the keys' affair


@pytest.mark.parametrize("name", ["eight_spilled", "four_spilled", "whole_256_masses_too"])
def test_keys_and_queries_without_finite_values(dev, name):  # noqa: F811
    """A NaN in a key of the last old row spoils the queries of its unit and the masses of the
    rows they see; one in a query's head that query, and the same masses; other units keep
    their bits."""
    p = next(p for p in mp.TOKENS + mp.PROMPTS if p.name == name)
    d, G = 128, p.Hq // p.Hkv
    clean, x = _pair(p, dev, d), _pair(p, dev, d)
    q, k, v = (_bf16(t, dev) for t in clean.inputs(p.n))
    want, out = (torch.zeros(q.shape, device=dev) for _ in range(2))
    clean.c.attend(q, want, d ** -0.5, k=k, v=v)
    q = q.clone()
    q[:, 1, p.n - 1, G, 0] = float("nan")  # head 0 of sequence 1's second unit
    nan = torch.zeros(q.shape[:-1], dtype=torch.bool, device=dev)
    nan[:, 1, p.n - 1, G] = True
    hit = torch.zeros(x.c.mass.shape, dtype=torch.bool, device=dev)
    for u, (unit, o) in enumerate(zip(x.units, x.off)):
        l, b, g = u // (p.B * p.Hkv), u // p.Hkv % p.B, u % p.Hkv
        if g == 3 and len(unit.K):
            x.c.k_pool[o + len(unit.K) - 1, 7] = float("nan")
            nan[l, b, :, 3 * G:4 * G] = True
            hit[o:o + len(unit.K) + p.n] = True
        if (b, g) == (1, 1):
            hit[o:o + len(unit.K) + p.n] = True
    x.c.attend(q, out, d ** -0.5, k=k, v=v)
    assert torch.equal(torch.isnan(out).all(dim=-1), nan) and torch.equal(torch.isnan(out).any(dim=-1), nan)
    same = ~nan
    same[:, 1, :, G:2 * G] = False  # (the maxima of a wave's columns follow one another)
    assert torch.equal(out[same], want[same])
    assert torch.equal(torch.isnan(x.c.mass), hit) and torch.equal(x.c.mass[~hit], clean.c.mass[~hit])
