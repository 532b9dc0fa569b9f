"""Appending many tokens at once (kv_append): four passes a wave for keys and values, and queries in
a launch of their own, sixteen passes a wave.  The pages and the queries hold bit for bit what the
same tokens give in calls of a few hundred, which take one pass a wave and are held against the
oracle elsewhere."""

import pytest

pytestmark = pytest.mark.gpu

CASES = [
    # tokens, q_heads, heads, dim, page, dtype, rot, pairs, norm, hadamard, code, queries apart
    (8209, 64, 8, 128, 64, "bfloat16", 96, "halves", True, True, {}, True),
    (8209, 66, 3, 128, 16, "float16", 128, "neighbours", True, True, dict(q=16, decoder=1), True),
    (8221, 128, 5, 64, 32, "bfloat16", 32, "neighbours", False, True, {}, True),
    (8193, 33, 1, 256, 256, "float16", 256, "halves", True, False, dict(q=7, k=3), True),
    (8200, 66, 1, 128, 64, "float32", 64, "halves", True, True, {}, True),
    (2057, 32, 8, 128, 64, "bfloat16", 128, "halves", True, True, {}, False),
    (8301, 4, 4, 64, 16, "float16", 64, "halves", True, True, {}, False),
    (2903, 6, 3, 256, 32, "bfloat16", 128, "neighbours", True, True, dict(values=dict(q=16)), False),
    (2903, 0, 3, 256, 32, "float16", 0, "halves", False, True, {}, False),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_many_tokens_equal_few(i, in_place):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_09720_amd as nq
    tokens, q_heads, heads, dim, page, dtype, rot, pairs, norm, hadamard, code, apart = CASES[i]
    assert tokens * heads * dim // 8 >= 1 << 18 or apart
    assert (tokens * q_heads * dim // 8 >= 1 << 23) == apart
    g = torch.Generator(device="cuda").manual_seed(i)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    rows = (rand(tokens, q_heads + 2 * heads, dim) * (0.1 + torch.rand(tokens, 1, 1, generator=g, device="cuda"))
            ).to(getattr(torch, dtype))
    pages = -(-tokens // page) + 2
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens]
    slots[::97] = -1                                             # left out of the cache
    slots[5::1001] = pages * page
    prep = dict(pairs=pairs, hadamard=hadamard)
    positions = None
    if rot:
        angle = 40 * torch.rand(3000, rot // 2, generator=g, device="cuda")
        prep.update(cos=angle.cos(), sin=angle.sin())
        positions = torch.randint(-5, 3005, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    if norm:
        prep.update(q_norm=1 + 0.2 * rand(dim), k_norm=1 + 0.2 * rand(dim))
    caches = [nq.kv_cache(pages, heads, dim, page, **code) for _ in range(2)]
    for c in caches:
        for t in (*c.k[:3], *c.v[:3]):
            t.zero_()
    q, k, v = rows.split((q_heads, heads, heads), 1)
    if not q_heads:
        q = None
    want = []
    for at in range(0, tokens, 311):
        part = slice(at, at + 311)
        want.append(nq.kv_append(caches[0], None if q is None else q[part], k[part], v[part], slots[part],
                                 positions=None if positions is None else positions[part], **prep))
    got = nq.kv_append(caches[1], q, k, v, slots, positions=positions, out=q if in_place else None, **prep)
    if q is not None:
        assert (got is q) == in_place
        assert torch.equal(got, torch.cat(want))
    for a, b in zip((*caches[0].k[:3], *caches[0].v[:3]), (*caches[1].k[:3], *caches[1].v[:3])):
        assert torch.equal(a, b)
    live = (slots >= 0) & (slots < pages * page)
    scales = caches[1].k.scales.view(pages, heads, page)
    assert int((scales > 0).sum()) == int(live.sum()) * heads
