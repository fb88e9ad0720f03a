"""The workspace of an 8-bit cache: what a program's calls leave behind stays bounded,
however many sizes and row bounds they come with."""


def test_what_is_kept(monkeypatch):
    import torch
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import Q8Cache
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    c = Q8Cache(1, 2, 28, 4, 128, [30000] * 8, "cpu")
    most = 0
    for n in list(range(1, 300)) + [1, 5]:
        for rows in (64 * n, 100 * n, 30000):
            need = vc.viscache_q8_attend_workspace_bytes(c.shape, n, rows)
            at, size = c._workspace(n, rows)
            assert size >= need and size == c._ws.numel() and at == c._ws.data_ptr()
            most = max(most, need)
    assert sum(x.numel() for x in c._kept) <= 4.5 * most  # three times the last, itself at most half more than needed
    for rows in range(20000):
        c._workspace(1, rows)
        assert len(c._ws_of) <= 4096
    assert sum(x.numel() for x in c._kept) <= 4.5 * most
