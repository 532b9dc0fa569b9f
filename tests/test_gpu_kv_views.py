"""Views that torch makes of a serving program's tensors, as arguments of kv_append and attend."""

import pytest

from test_gpu_attend import nq  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


def test_strides_of_a_single_token_or_head(nq):
    """A dimension of one entry may have any stride: a token of a row of odd width, a head alone."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    lengths, table = torch.tensor([5], dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    slot = torch.tensor([4], device="cuda")
    for heads in (2, 1):
        caches = [nq.kv_cache(1, heads, 64, 16) for _ in range(2)]
        past = rand(4, heads, 64)
        for c in caches:
            nq.kv_append(c, None, past, past, torch.arange(4, device="cuda"))
        rows = rand(1, 6 * heads * 64)
        odd = rand(1, 6 * heads * 64 + 3)[:, :-3]                # a row 3 entries wider than the heads
        odd.copy_(rows)
        outs = []
        for c, x in ((caches[0], rows), (caches[1], odd)):
            q, k, v = x.unflatten(1, (6 * heads, 64)).split((4 * heads, heads, heads), 1)
            if heads == 1 and x is odd:
                k, v = (t.as_strided(t.shape, (t.stride(0), 7, 1)) for t in (k, v))
            q = nq.kv_append(c, q, k, v, slot)
            one = q if x is not odd else q.as_strided(q.shape, (1, *q.stride()[1:]))
            outs.append(nq.attend(c, one, table, lengths))
        assert torch.equal(*outs)


def test_one_table_row_for_all_sequences(nq):
    """Sequences over the same pages, their table an expanded row."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = nq.kv_cache(8, 2, 64, 16)
    k, v = (torch.randn(100, 2, 64, generator=g, device="cuda") for _ in range(2))
    nq.kv_append(cache, None, k, v, torch.arange(100, device="cuda"))
    q = torch.randn(3, 4, 64, generator=g, device="cuda")
    lengths = torch.tensor([100, 77, 3], dtype=torch.int32, device="cuda")
    row = torch.arange(8, dtype=torch.int32, device="cuda").view(1, 8)
    want = nq.attend(cache, q, row.repeat(3, 1), lengths)
    assert torch.equal(nq.attend(cache, q, row.expand(3, -1), lengths), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = nq.attend(cache, q, row.expand(3, -1), lengths, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
