"""Attention of one new token over a cache with infinite values and with values of the largest size."""
import math

import numpy as np
import pytest

from oracle import cache_oracle as co
from paper_2509_19836_amd import workloads as wl
from tests import test_gpu_paged_cache as tp

pytestmark = pytest.mark.gpu

# (kv_heads, bound of the rows): a work-group for each (sequence, key head); rows dealt; dealt to work-groups of several heads
MODES = {"direct": (4, 500), "dealt": (3, 40000), "beside": (4, 300000)}


def bound_of(mode, page_rows):
    """The mode's bound, in whole pages."""
    rows = MODES[mode][1]
    return rows // page_rows * page_rows


@pytest.mark.parametrize("page_rows", [16, 5])
@pytest.mark.parametrize("group", [2, 20])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", list(MODES))
def test_infinite_values_stay_infinite(lib, mode, d, group, page_rows):
    """A value's infinity is its element's result for every head that gives it a weight, whatever that weight's bits are (a power of two, as with a
    query of zeros, among them); infinities of both signs in an element make it NaN; other elements are as without."""
    import torch
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90000 + d + group + page_rows))
    Hkv, bound = MODES[mode][0], bound_of(mode, page_rows)
    rows = [300, 41]
    P = tp.Paged(lib, rng, rows, page_rows, Hkv, d, cols=bound // page_rows)
    q, q_host = tp.queries(rng, 2, Hkv * group, d)
    q[1], q_host[1] = 0, 0
    shares, heads, direct = lib.burst_attn_decode_plan(lib.shape(2, Hkv * group, Hkv, d, 1, bound, d ** -0.5), P.cache)
    assert direct == (mode == "direct") and (heads > 1) == (mode == "beside")
    for b, places in enumerate((((299, 3, math.inf), (17, 9, -math.inf), (0, 20, math.inf), (160, 20, -math.inf)),
                                ((40, 3, math.inf), (3, 9, -math.inf), (32, 20, math.inf), (31, 20, -math.inf)))):
        for t, j, x in places:
            page, r = co.slots(P.table, page_rows, b, t)
            P.dev["v"][page, r, :, j], P.host["v"][page, r, :, j] = x, 0.0
    print(f"infinite values, {mode} d={d} group={group} pages of {page_rows}", flush=True)
    o, lse = tp.run_decode(lib, P, q, d ** -0.5, bound)
    assert (o[..., 3] == math.inf).all() and (o[..., 9] == -math.inf).all() and torch.isnan(o[..., 20]).all()
    o[..., [3, 9, 20]] = 0.0
    ref = P.decode(q_host, d ** -0.5)
    for x in (ref[0], ref[2]):
        x[..., [3, 9, 20]] = 0.0
    tp.check_decode(o, lse, ref, 300, d)


@pytest.mark.parametrize("mode", list(MODES))
def test_rows_without_weight_have_no_share(lib, mode):
    """Rows whose weight fp32 does not hold, with the largest values that bf16 has: O is that of the others."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90050))
    Hkv, bound = MODES[mode][0], bound_of(mode, 16)
    P = tp.Paged(lib, rng, [333], 16, Hkv, 128, cols=bound // 16)
    q, q_host = tp.queries(rng, 1, 2 * Hkv, 128)
    q[..., 5], q_host[..., 5] = 2.0, 2.0
    for t in (0, 31, 100, 332):
        page, r = co.slots(P.table, 16, 0, t)
        P.dev["k"][page, r, :, 5] = -4096.0                                 # (times 2 and the scale: 724 below the others)
        P.dev["v"][page, r, :, 64:] = 3e38
    P.refresh()
    o, lse = tp.run_decode(lib, P, q, 128 ** -0.5, bound)
    O, lse_ref, weight, _ = P.decode(q_host, 128 ** -0.5)                   # (weights of 0 in 64 bits, next to nothing)
    for t in (0, 31, 100, 332):
        page, r = co.slots(P.table, 16, 0, t)
        P.host["k"][page, r] = 0.0
    size = P.decode(q_host, 128 ** -0.5)[3]                                 # the tolerance goes by the scores of the others
    tp.check_decode(o, lse, (O, lse_ref, weight, size), 333, 128)


@pytest.mark.parametrize("place", [0, 250, 399])
@pytest.mark.parametrize("mode", list(MODES))
def test_infinite_values_of_small_weight(lib, mode, place):
    """A weight of 2^-86 of the others', before them, among them and behind them: the infinity is there all the same."""
    rng = np.random.Generator(np.random.PCG64(wl.BASE_SEED + 90060 + place))
    Hkv, bound = MODES[mode][0], bound_of(mode, 16)
    P = tp.Paged(lib, rng, [400], 16, Hkv, 64, cols=bound // 16)
    P.dev["k"].zero_()
    page, r = co.slots(P.table, 16, 0, place)
    P.dev["k"][page, r, :, 11] = -60.0                                      # (e^-60 = 2^-86.6)
    P.dev["v"][page, r, :, 3], P.dev["v"][page, r, :, 9] = math.inf, -math.inf
    q, _ = tp.queries(rng, 1, 3 * Hkv, 64)
    q[..., 11] = 1.0
    o, lse = tp.run_decode(lib, P, q, 1.0, bound)
    assert (o[..., 3] == math.inf).all() and (o[..., 9] == -math.inf).all()
    o[..., [3, 9]] = 0.0
    assert o.isfinite().all() and np.abs(lse.cpu().numpy() - math.log(399)).max() <= 1e-5
