"""Attention over a coded KV cache (attend) at the accuracy of its contract: weights of 22 bits for
every type and number of queries.

The bound is that of test_gpu_attend.py with 22-bit weights throughout (the second term of a weight
is there for 16-bit queries of many rows as well): an output of n tokens is off by at most
(2 d + 2^-22 + (n + 64) 2^-22) sum_j p_j |V_j| + f R sum_j |V_j| / r_j / L + u |exact| + half the type's
smallest step, with d the error of a score, f = 2^-37 and R the largest scale r of a value.
"""

import numpy as np
import pytest

from test_gpu_attend import MANY, SHAPES, SUBNORMAL, ULP, Call, nq  # noqa: F401 (nq: the fixture)

pytestmark = pytest.mark.gpu


class Exact(Call):
    """A call whose bounds are those above, and whose value scales can be changed."""

    def __init__(self, *args, **more):
        super().__init__(*args, **more)
        self.U = self.V / self.r               # the values without their scales

    def largest(self, e, r):
        """R, from the exponentials relative to a row's largest and the scales."""
        return r.max(initial=0.0)

    def exact(self):
        T, H = self.q64.shape[:2]
        out, bound = np.zeros(self.q64.shape), np.zeros(self.q64.shape)
        lse, lse_bound = np.full((T, H), -np.inf), np.zeros((T, H))
        for b in range(len(self.lengths)):
            lo, hi = self.starts[b], self.starts[b + 1]
            n = int(self.lengths[b])
            p = np.arange(n - (hi - lo), n)[:, None]
            j = np.arange(n)
            see = j <= p
            if self.window:
                see &= (j > p - self.window) | (j < self.sinks)
            for h in range(self.heads):
                K, ok = self.rows(self.K, b, h)
                U, _ = self.rows(self.U, b, h)
                r = self.rows(self.r, b, h)[0][:, 0]
                s_ = see & ok
                for hq in range(h * self.group, (h + 1) * self.group):
                    q = self.q64[lo:hi, hq]
                    s = np.where(s_, self.scale * q @ K.T, -np.inf)
                    size = np.where(s_, abs(self.scale) * np.abs(q) @ np.abs(K).T, 0.0).max(-1, initial=0.0)
                    any_ = s_.any(-1)
                    top = np.where(any_, s.max(-1, initial=-np.inf), 0.0)
                    e = np.exp(s - top[:, None])
                    total = np.where(any_, e.sum(-1), 1.0)
                    w = e / total[:, None] * r
                    out[lo:hi, hq] = w @ U
                    R = self.largest(e, r) / total[:, None]
                    d = (self.dim + 8) * 2.0 ** -22 * size
                    rel = 2 * d + 2.0 ** -22 + (n + 64) * 2.0 ** -22
                    bound[lo:hi, hq] = rel[:, None] * (w @ np.abs(U)) + 2.0 ** -37 * R * (s_ @ np.abs(U))
                    lse[lo:hi, hq] = np.where(any_, top + np.log(total), -np.inf)
                    lse_bound[lo:hi, hq] = d + (n + 64) * 2.0 ** -22 + 2.0 ** -22 * np.abs(top)
        return out, lse, bound + ULP[self.dtype] * np.abs(out) + SUBNORMAL[self.dtype], lse_bound


@pytest.mark.parametrize("i", [i for i, case in enumerate(MANY) if case[2].get("dtype") != "f32"])
def test_prompts_of_16_bits(nq, i):
    lengths, counts, more = MANY[i]
    Exact(nq, 500 + i, lengths, counts, **more).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_prompt_of_one_query_more(nq, dtype):
    """The same rows in a call of 64 rows a KV head and in one of 68: within both bounds."""
    c = Exact(nq, 530, [900], [17], dtype=dtype)
    c.check()
    c.q, c.q64 = c.q[1:], c.q64[1:]
    c.starts[1] -= 1
    c.check()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_that_are_all_not_numbers(nq, shape, dtype):
    """A query that is not a number, or whose only token's key is not, gives outputs that are not
    numbers (and not those of a query that sees nothing), and reaches no other row."""
    import torch
    lengths, counts, more = shape
    c = Exact(nq, 540, lengths, counts, dtype=dtype, **more)
    lse, kept = (torch.empty(c.q.shape[:2], device="cuda") for _ in range(2))
    ref = c.run(lse=kept)
    hit = torch.zeros(c.q.shape[:2], dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[0, 0] = True
    q = c.q.clone()
    q[hit, 5] = float("nan")
    got = c.run(q=q, lse=lse)
    assert torch.isnan(got[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(got[~hit], ref[~hit]) and torch.equal(lse[~hit], kept[~hit])
    # token 0's key of KV head 0: all that the query at position 0 sees
    c = Exact(nq, 542, counts, counts, dtype=dtype, **more)
    c.cache.k.scales[int(c.table[0, 0]) * c.heads * c.page] = float("nan")
    got = c.run(lse=lse)
    assert torch.isnan(got[:counts[0], :c.group]).all() and torch.isnan(lse[:counts[0], :c.group]).all()
    assert torch.isfinite(got[:, c.group:]).all() and torch.isfinite(lse[:, c.group:]).all()


class Seen(Exact):
    """With R the largest product of a weight and its value's scale among the tokens that a row
    sees, relative to the row's largest weight."""

    def largest(self, e, r):
        return (e * r).max(-1, initial=0.0, keepdims=True)


def scaled(c, b, tokens, factor):
    """Multiplies the value scales of tokens of sequence b, in the cache and in the reference."""
    for t in tokens:
        page, slot = int(c.table[b, t // c.page]), t % c.page
        for h in range(c.heads):
            row = (page * c.heads + h) * c.page + slot
            c.r[page, h, slot] *= factor
            c.cache.v.scales[row] = float(c.r[page, h, slot, 0])
    c.r[:] = c.cache.v.scales.double().cpu().numpy().reshape(c.r.shape)


HIDDEN = [
    # lengths, counts, more, sequence, tokens that some or all queries do not see
    ([195, 70], [1, 1], dict(window=40, sinks=2), 0, [5, 150]),          # in tiles with seen tokens
    ([195, 70], [1, 1], dict(window=40, sinks=2, dim=64, group=20, heads=1), 0, [5, 150]),
    ([300, 1040], [4, 5], dict(dim=256, group=2), 1, [1037, 1038]),      # drafted: after some queries
    ([300, 21], [4, 5], dict(group=12, heads=1), 0, [298]),              # two row blocks
    ([200, 90], [70, 66], dict(group=2), 0, [140, 180, 199]),            # a prompt's later tokens
    ([200, 90], [200, 90], dict(group=1, dim=64), 0, [3, 63, 64, 130]),
    ([400, 150], [100, 150], dict(window=30, sinks=3), 0, [5, 300, 331, 399]),
    ([140, 70], [80, 33], dict(dim=256, group=2, heads=1), 0, [90, 139]),
    ([1500, 700], [30, 33], dict(dim=64, group=5, heads=1), 0, [1490]),  # chunks along the cache
]


@pytest.mark.parametrize("factor", [2.0 ** 12, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(HIDDEN)))
def test_large_scales_that_are_not_seen(nq, i, dtype, factor):
    """A value of large finite scale has no part in the rows that do not see its token."""
    lengths, counts, more, b, tokens = HIDDEN[i]
    c = Seen(nq, 560 + i, lengths, counts, dtype=dtype, **more)
    scaled(c, b, tokens, factor)
    c.check()


@pytest.mark.parametrize("factor", [2.0 ** 20, 2.0 ** 40, 2.0 ** -40])
@pytest.mark.parametrize("shape", [([150, 90], [2, 1], {}), ([150, 90], [70, 80], dict(group=1)),
                                   ([1000, 90], [1, 1], dict(dim=64))])
def test_large_scales_of_little_weight(nq, shape, factor):
    """Scores tens apart: what a token's scale does is what its weight leaves of it, row by row,
    whether the weight of a large scale is next to nothing or a small scale has all the weight."""
    lengths, counts, more = shape
    c = Seen(nq, 580, lengths, counts, dtype="f32", scale=0.4, spread=3.0, **more)
    scaled(c, 0, range(0, lengths[0], 7), factor)
    c.check()


@pytest.mark.parametrize("factor", [2.0 ** -100, 2.0 ** -60, 2.0 ** 35, 2.0 ** 60, 2.0 ** 110])
@pytest.mark.parametrize("shape", [([391, 90], [1, 1], {}), ([150, 90], [70, 80], dict(group=1, window=50))])
def test_scales_anywhere_in_fp32(nq, shape, factor):
    """Values of any size have the same relative errors and leave the sums as they are."""
    lengths, counts, more = shape
    c = Seen(nq, 590, lengths, counts, dtype="f32", **more)
    for b, n in enumerate(lengths):
        scaled(c, b, range(n), factor)
    c.check()


@pytest.mark.parametrize("shape", [([391, 90], [1, 1], {}), ([150, 90], [70, 80], dict(group=1))])
def test_scales_of_zero(nq, shape):
    """Rows of zeros among the values and nothing but such rows."""
    import torch
    lengths, counts, more = shape
    c = Seen(nq, 595, lengths, counts, dtype="f32", **more)
    scaled(c, 0, range(0, lengths[0], 3), 0.0)
    c.check()
    scaled(c, 0, range(lengths[0]), 0.0)
    got = c.check()
    assert not torch.any(got[:counts[0]]).item()


@pytest.mark.parametrize("shape", [([195, 70], [2, 1], dict(window=40, sinks=2)), ([200, 90], [70, 66], dict(group=2))])
def test_rows_do_not_depend_on_other_rows(nq, shape):
    """A row's bits are the same whatever the queries beside it are."""
    import torch
    lengths, counts, more = shape
    c = Seen(nq, 598, lengths, counts, **more)
    ref = c.run()
    q = c.q.clone()
    q[0, 1::2] *= 40.0
    q[1] = 0.0
    got = c.run(q=q)
    same = torch.ones(q.shape[:2], dtype=torch.bool, device="cuda")
    same[0, 1::2] = same[1] = False
    assert torch.equal(got[same], ref[same])
