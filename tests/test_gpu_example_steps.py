"""The example's layer step by step: what each of its calls returns against 64-bit arithmetic on the
operands that the codes stand for, so that the layer's distance from the uncoded one is that of its
codes and nothing else.

Bounds, relative to the norm of the whole result: products of decoded operands hold them exactly or
to 2^-9 an entry (bf16 tiles) and add in fp32, so 2^-8 is beyond them; attention's outputs are rounded
to bf16 (2^-9) after scores of fp32 sums over 128 entries, so 2^-8 as well.
"""

import os
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def near(got, want, bound):
    error = float((got.double() - want).norm() / want.norm())
    assert error <= bound, error


def test_the_layers_steps():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import coded_attention
    finally:
        sys.path.pop(0)
    nq, seen = coded_attention.nq, []

    class Recording:
        """The package, keeping the attention's and the products' arguments and results."""

        def __getattr__(self, name):
            f = getattr(nq, name)
            if name not in ("attend", "encode_matmul", "kv_append"):
                return f

            def call(*args, **more):
                out = f(*args, **more)
                seen.append((name, args, more, out))
                return out
            return call
    q_heads, heads, dim, hidden = 8, 2, 128, 4096
    layer = coded_attention.CodedAttention(hidden, q_heads, heads, dim, pages=12, positions=512)
    g = torch.Generator(device="cuda").manual_seed(3)
    table = torch.randperm(12, generator=g, device="cuda").to(torch.int32).view(2, 6)
    coded_attention.nq = Recording()
    try:
        lengths = [0, 0]
        for counts in ([150, 77], [1, 1], [3, 1]):
            lengths = [n + c for n, c in zip(lengths, counts)]
            x = torch.randn(sum(counts), hidden, generator=g, device="cuda").bfloat16()
            seen.clear()
            y = layer(x, table, lengths, counts)
            (_, _, _, (a, qkv)), (_, _, _, q), (_, args, more, out), (_, _, _, (b, last)) = seen
            assert [s[0] for s in seen] == ["encode_matmul", "kv_append", "attend", "encode_matmul"]
            near(qkv, nq.decode(a).double() @ nq.decode(layer.qkv).double().t(), 2.0 ** -8)
            near(last, nq.decode(b).double() @ nq.decode(layer.o).double().t(), 2.0 ** -8)
            assert y is last and args[1] is q
            # rotating x and w alike leaves their products: the coded operands are the rotated rows
            near(nq.decode(a), nq.rotate(x).double(), 0.12)
            assert all(torch.equal(s, t) for s, t in zip(b[:3], nq.encode(out.flatten(1), rotate=True)[:3]))
            # attention over the rows that the cache stands for, keys and values of this layer's product
            rows = qkv.bfloat16().view(len(x), -1, dim)
            pools = [nq.decode(p).double().view(12, heads, 64, dim) for p in (layer.cache.k, layer.cache.v)]
            at = 0
            for s, (n, c) in enumerate(zip(lengths, counts)):
                K, V = (p[table[s, :-(-n // 64)].long()].transpose(1, 2).reshape(-1, heads, dim)[:n] for p in pools)
                near(V[n - c:], rows[at:at + c, q_heads + heads:].double(), 0.12)
                p = torch.arange(n - c, n, device="cuda").unsqueeze(1)
                hidden_ones = torch.arange(n, device="cuda") > p
                for h in range(q_heads):
                    kv = h // (q_heads // heads)
                    score = (q[at:at + c, h].double() @ K[:, kv].t()) * dim ** -0.5
                    want = torch.softmax(score.masked_fill(hidden_ones, float("-inf")), -1) @ V[:, kv]
                    near(out[at:at + c, h], want, 2.0 ** -8)
                at += c
    finally:
        coded_attention.nq = nq
