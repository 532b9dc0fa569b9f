"""Bounds of a call over a coded KV cache that are looser than what is there: no tokens at all, more
queries a sequence than the call has, workspaces sized for larger calls."""

import pytest

from test_gpu_attend import Call, nq  # noqa: F401 (nq: the fixture)

pytestmark = pytest.mark.gpu


def test_no_tokens(nq):
    """A batch that has run empty is a no-op, with or without starts."""
    import torch
    cache = nq.kv_cache(2, 2, 64, 16)
    q = torch.empty(0, 4, 64, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    starts = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert nq.attend(cache, q, torch.empty(0, 2, dtype=torch.int32, device="cuda"), none).shape == q.shape
    table, lengths = torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    assert nq.attend(cache, q, table, lengths, starts=starts, max_queries=4).shape == q.shape
    assert nq.attend_workspace_size(cache, 0, 4, 3, max_queries=4, max_length=32) == 0


def test_more_queries_allowed_than_there_are(nq):
    """A fixed bound, such as the number of drafted tokens, also where fewer rows are left."""
    import torch
    c = Call(nq, 700, [90, 40], [1, 2], dtype="f32")
    assert torch.equal(c.run(max_queries=50), c.run(max_queries=3))
    c.check(max_queries=50)


def test_one_workspace_for_smaller_calls(nq):
    """A workspace of the largest call's size is the one that smaller calls use, whether they are
    split more or less: nothing is allocated beside it."""
    import torch
    heads, group, dim, most = 8, 4, 128, 2049
    calls = [([2049], [1]), ([2048], [1]), ([300], [1]), ([2048], [17]), ([2040], [40]), ([1500], [300]),
             ([129], [2])]
    ws = None
    for i, (lengths, counts) in enumerate(calls):
        c = Call(nq, 710 + i, lengths, counts, heads=heads, group=group, dim=dim, page=64, dtype="f32")
        if ws is None:
            need = nq.attend_workspace_size(c.cache, 300, heads * group, 1, max_queries=300, max_length=most)
            ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        up = lambda a: torch.from_numpy(a).cuda()
        args = (c.cache, c.q, up(c.table), up(c.lengths))
        more = dict(starts=up(c.starts), max_queries=counts[0], max_length=lengths[0], out=torch.empty_like(c.q),
                    workspace=ws)
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        got = nq.attend(*args, **more)
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
        assert torch.equal(got, c.run())
