"""The norm of kv_append on rows that hold an infinity or are not numbers, and on rows of zeros without
eps: entry by entry what its formula gives, x <- fl32(fl32(x f) w) with f = fl32(1 / sqrt(mean + eps))
(an infinite entry makes f 0: it becomes NaN itself and the others 0)."""

import numpy as np
import pytest

from test_gpu_kv_cache import nq, prepared, torch_dtype  # noqa: F401 (nq: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e-5, 0.0])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_that_are_not_finite(nq, dim, dtype, eps):
    import torch
    g = torch.Generator(device="cuda").manual_seed(dim)
    q = torch.randn(9, 3, dim, generator=g, device="cuda").to(torch_dtype(dtype))
    k = torch.randn(9, 1, dim, generator=g, device="cuda").to(q.dtype)
    q[0, 0, 5] = float("inf")
    q[2, 1, [3, dim - 1]] = torch.tensor([float("-inf"), float("inf")], device="cuda").to(q.dtype)
    q[4, 2, 7] = float("nan")
    q[5, 0] = 0.0
    w = 1 + 0.2 * torch.randn(dim, generator=g, device="cuda")
    cache = nq.kv_cache(1, 1, dim, 16)
    got = nq.kv_append(cache, q, k, k, torch.arange(9, device="cuda"), q_norm=w, k_norm=w, eps=eps, hadamard=False)
    with np.errstate(invalid="ignore", divide="ignore"):
        want = prepared(q.float().cpu().numpy(), w.cpu().numpy(), eps, None, None, None, None, False)
    want = torch.from_numpy(want).to(q.dtype).float().numpy()
    assert np.array_equal(got.float().cpu().numpy(), want, equal_nan=True)
    bad = np.isnan(want)
    assert bad[0, 0].sum() == 1 and bad[2, 1].sum() == 2 and bad[4, 2].all()
    assert bad[5, 0].all() == (eps == 0.0)
