"""Attention over 8-bit caches in which every block counts (tests/q8_blocks.py): on
the CPU, that the loss or the doubling of any block is past the tolerance of a row that
is looked at; on the GPU, the outputs."""
import numpy as np
import pytest

from tests import q8_blocks as qb
from tests import q8_ref as ref

FMTS = ("int8", "e4m3")


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("case", qb.CASES, ids=lambda c: c.name)
def test_no_block_may_go_unseen(case, fmt):
    """Every block of which a sampled query sees 16 rows or more, at the wider tolerance of
    bf16 outputs.  (A unit's only block may be taken twice: that is the same output.)"""
    K, V, q = qb.data(case)
    if case.name.startswith("whole") and len(K) > 20:
        units = range(0, len(K), 11)
    else:
        units = range(len(K))
    for u in units:
        found, needed = set(), set()
        for _, want, tol, moved, seen in qb.expected(case, ref.read_back(K[u], fmt), ref.read_back(V[u], fmt), q, u,
                                                     False, blocks=True):
            if moved is None:
                continue
            for kind in range(2 if len(seen) > 1 else 1):
                past = (np.abs(moved[kind] - want) > tol).any(axis=(1, 2))
                needed |= {(kind, j) for j in np.flatnonzero(seen >= 16)}
                found |= {(kind, j) for j in np.flatnonzero(past)}
        assert needed <= found, (u, sorted(needed - found)[:5])


def test_cases_are_cut_as_they_say():
    """Partial results take most of a workspace; without them there is a word a unit."""
    import paper_2608_24063_amd as vc
    for c in qb.CASES:
        shape = vc.vc_decode_shape(c.B, c.L, c.G * c.Hkv, c.Hkv, c.d)
        need = vc.viscache_q8_attend_workspace_bytes(shape, c.n, max(c.lens) if c.most is None else c.most)
        assert (need > 4 * len(c.lens) + 256) == c.cut, c.name


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("case", qb.CASES, ids=lambda c: c.name)
def test_every_block_counts(case, fp32, fmt):
    import paper_2608_24063_amd as vc
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_24063_amd.tensors import Q8Cache
    dev = torch.device("cuda:0")
    L, B, Hkv, d = case.L, case.B, case.Hkv, case.d
    K, V, q = qb.data(case)
    c = Q8Cache(L, B, case.G * Hkv, Hkv, d, case.lens, dev, format=fmt)
    t = lambda x: torch.from_numpy(x).to(dev).to(torch.bfloat16)  # noqa: E731
    rows = [t(np.concatenate(x)) for x in (K, V)]
    off = torch.from_numpy(np.concatenate(([0], np.cumsum(case.lens)[:-1])).astype(np.int64) * d).to(dev)
    one = vc.vc_decode_shape(len(K), 1, 1, 1, d)  # a unit a sequence: counts of their own
    cnt = torch.tensor(case.lens, dtype=torch.int32, device=dev)
    vc.viscache_q8_append(one, c.c, *[vc.vc_rows(x.data_ptr(), 0, 0, d, 0) for x in rows], max(case.lens), cnt.data_ptr(),
                          off.data_ptr(), torch.cuda.current_stream().cuda_stream)
    out = torch.full(q.shape, 7.0, dtype=torch.float32 if fp32 else torch.bfloat16, device=dev)
    counts = torch.tensor(case.counts, dtype=torch.int32, device=dev) if case.ragged else None
    c.attend(t(q), out, d ** -0.5, count=counts, causal=case.causal, max_rows=case.most)
    got = out.float().cpu().numpy()
    for u in range(len(K)):
        l, b, g = u // (B * Hkv), u // Hkv % B, u % Hkv
        assert (got[l, b, min(max(case.counts[b], 0), case.n):] == 7.0).all()
        for i, want, tol, _, _ in qb.expected(case, ref.read_back(K[u], fmt), ref.read_back(V[u], fmt), q, u, fp32):
            err = np.abs(got[l, b, i, g * case.G:(g + 1) * case.G] - want)
            assert (err <= tol).all(), (u, i, float((err / np.maximum(tol, 1e-30)).max()))
