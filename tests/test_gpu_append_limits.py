"""Appending to a paged cache at its limits: scales of e4m3 at both ends of fp32, and more tokens than one launch has threads for."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from tests import test_gpu_paged_cache as tp

pytestmark = pytest.mark.gpu


def test_scales_of_all_sizes(lib):
    """Any positive scale, those whose reciprocal fp32 does not hold among them (a head of zeros over the least scale that a program allows): number / scale
    rounded to e4m3.  Tolerance: two roundings of the division and half a step (2^-10 at the bottom)."""
    import torch
    scales = np.array([2.0 ** -149, 2.0 ** -140, 3e-41, 2.0 ** -127, 1.2e-38, 2.0 ** -101, 2.0 ** -99, 1.0, 3.0, 2.0 ** 99, 2.0 ** 101, 2.0 ** 126, 3e38], np.float32)
    H, d, n = scales.size, 64, 5
    P = tp.Paged(lib, np.random.Generator(np.random.PCG64(12)), [n], 16, H, d, f8=True)
    for i in (4, 5):
        P.cache._tensors[i].copy_(torch.from_numpy(scales).cuda())
    rng = np.random.Generator(np.random.PCG64(13))
    with np.errstate(over="ignore"):
        x = (rng.standard_normal((1, n, H, d)) * 100.0 * scales.astype(np.float64)[:, None]).clip(-3e38, 3e38)
    x[..., 0], x[..., 1], x[..., 2], x[..., 3] = 0.0, -0.0, 1.0, 1e38
    k = torch.from_numpy(x).float().to(torch.bfloat16)
    host = k.double().numpy()
    k = k.cuda()
    lib.burst_attn_cache_append(lib.shape(1, H, H, d, n, 0, 1.0), P.cache, k, k)
    page, r = co.slots(P.table, 16, 0, np.arange(n))
    want = np.clip(host[0] / scales.astype(np.float64)[:, None], -448.0, 448.0)
    tol = 3 * 2.0 ** -24 * np.abs(want) + np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10)
    P.refresh()
    for name in "kv":
        got = P.host[name][page, r]
        assert np.isfinite(got).all(), scales[np.nonzero(~np.isfinite(got))[1]]
        assert (np.abs(got - want) <= tol).all(), scales[np.unique(np.nonzero(np.abs(got - want) > tol)[1])]


def test_more_tokens_than_a_launch_has_threads_for(lib):
    """A padded batch of 3 x 2^28 tokens, few of them new: the rows of a sequence whose tokens two launches share, and of one behind."""
    import torch
    d, sq = 128, (1 << 28) - 100
    P = tp.Paged(lib, np.random.Generator(np.random.PCG64(14)), [20, 150, 30], 16, 1, d)
    k, v = (torch.randn(3, 1, 1, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    new = torch.tensor([0, 150, 3], dtype=torch.int32, device="cuda")
    lib.burst_attn_cache_append(lib.shape(3, 1, 1, d, sq, 0, 1.0), P.cache, k.expand(3, sq, 1, d), v.expand(3, sq, 1, d), new)
    before = dict(P.host)
    P.refresh()
    for name, x in (("k", k), ("v", v)):
        x = x.double().cpu().numpy()
        assert np.array_equal(P.host[name], co.append(before[name], np.broadcast_to(x, (3, 150, 1, d)), P.table, [20, 150, 30], [0, 150, 3]))
