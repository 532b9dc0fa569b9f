"""What kv_append and attend allocate for a call on another stream comes from that stream's memory:
blocks that the current stream has freed, whose last uses may still be queued there, are not taken
for it, and its own are not handed out to the current stream while it runs."""

import pytest

pytestmark = pytest.mark.gpu


def test_memory_of_a_call_on_another_stream():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_09720_amd as nq
    cache = nq.kv_cache(64, 2, 128, 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1000, h, 128, generator=g, device="cuda") for h in (8, 2, 2))
    slots = torch.arange(1000, device="cuda")
    table = torch.arange(64, dtype=torch.int32, device="cuda").view(1, 64)
    lengths, starts = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([1000], [0, 1000]))
    ref = nq.kv_append(cache, q, k, v, slots)
    want = nq.attend(cache, ref, table, lengths, starts=starts)
    need = nq.attend_workspace_size(cache, 1000, 8, 1, max_queries=1000, max_length=1024)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    # blocks that the current stream has freed, of the sizes that the calls need
    torch.cuda.empty_cache()
    freed = [torch.empty_like(q) for _ in range(4)] + [torch.empty(n, dtype=torch.uint8, device="cuda")
                                                       for n in (need, need, q.numel() * 16)]
    spans = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in freed]
    del freed
    turned = nq.kv_append(cache, q, k, v, slots, stream=side)
    out = nq.attend(cache, turned, table, lengths, starts=starts, stream=side)
    side.synchronize()
    assert torch.equal(turned, ref) and torch.equal(out, want)
    for t in (turned, out):
        assert not any(lo < t.data_ptr() + t.numel() * 4 and t.data_ptr() < hi for lo, hi in spans)
    # and back: the side stream's blocks stay its own
    kept = [t.data_ptr() for t in (turned, out)]
    del turned, out
    assert not any(torch.empty_like(q).data_ptr() in kept for _ in range(4))
